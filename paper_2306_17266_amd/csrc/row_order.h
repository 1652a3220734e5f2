// What sampling (sample.hip) and the top logits (top_logits.hip) share: the last kept position of a row's order.
//
// Both need it: the first position at which the number of logits reaches k or (sampling) their summed weight reaches top_p of the
// row's sum.  No row is sorted for it.  The range of keys that holds the position is cut finer by histograms over the keys until
// a wave can rank what is left, or one key is left.
//
// Sums of weights are whole numbers (fixed point in 64 bits): the same in whatever order atomics in LDS make them, so that a class
// whose interval of the sum is hit by the random number is the same in every run.  Which class that is is decided next to borders,
// so a weight has more than 32 bits: 24 would let one draw in a few hundred rows of 100 000 logits go to a neighbour.
#pragma once

#include "logits_device.h"

namespace sushi {

typedef unsigned long long u64;

constexpr double LN2 = 6.931471805599453094e-01;
constexpr int MEMBERS = 64;  // that one wave ranks, a lane each

struct SearchLds {
    u64 weight[BINS + 1];  // (the last: of what is in no order)
    uint32_t count[BINS];
    u64 member[MEMBERS];  // keys above indexes
    u64 part64[16];
    uint32_t part32[16];
    float part_f[16];
    int bin;  // what find_bin() found: the interval, what lies before it, its members
    uint32_t before, inside;
    u64 weight_before;
    int n, rank;
};

// The last kept position of an order.
struct Cut {
    uint32_t key;
    int index;
    __device__ __forceinline__ bool keeps(uint32_t k, int j) const { return k > key || (k == key && j <= index); }
};
__device__ __forceinline__ Cut keep_all() { return Cut{KEY_NONE + 1, 0x7FFFFFFF}; }

// A weight as a whole number of 2^-fraction (fraction <= 50), rounded: 2^52 is added, the number stands in the low bits.
__device__ __forceinline__ u64 fixed_weight(double t, int fraction) {
    return (u64)__double_as_longlong(ldexp(exp2_64<11>(t), fraction) + 4503599627370496.0) & ((1ull << 52) - 1);
}
__device__ __forceinline__ int bits_of(int n) { return n > 1 ? 32 - __builtin_clz(n - 1) : 0; }  // n <= 2^bits_of(n)
// Bits behind the point for sums of n weights: below 2^63.
__device__ __forceinline__ int fraction_bits(int n) { return min(62 - bits_of(n), 50); }

// When the order is cut: at the first position where this many logits, or this weight, has been reached.
struct Limit {
    uint32_t count;
    double weight;
    __device__ __forceinline__ bool reached(uint32_t n, u64 w) const { return n >= count || (double)w >= weight; }
};

// Finds the interval in which the limit is reached, counting from (s.before, s.weight_before); s.bin = -1: in none.  n, w: this
// thread's run of intervals, their members and weights.  share >= 0: that share of all weights is the limit's.  From interval `stop` on the
// limit counts as reached.
template <int THREADS>
__device__ void find_bin(SearchLds &s, Limit &limit, float share, const uint32_t (&n)[BINS / THREADS], const u64 (&w)[BINS / THREADS], int stop = BINS) {
    constexpr int OWN = BINS / THREADS, WAVES = THREADS / 64;
    const int tid = threadIdx.x, wave = tid >> 6;
    uint32_t n_before = s.before, n_own = 0;
    u64 w_before = s.weight_before, w_own = 0;
#pragma unroll
    for (int b = 0; b < OWN; ++b) n_own += n[b], w_own += w[b];
    const uint32_t n_upto = wave_scan(n_own);
    const u64 w_upto = wave_scan(w_own);
    if ((tid & 63) == 63) s.part32[wave] = n_upto, s.part64[wave] = w_upto;
    if (tid == 0) s.bin = -1;
    __syncthreads();
    n_before += sum_before<WAVES>(s.part32) + n_upto - n_own;
    w_before += sum_before<WAVES>(s.part64) + w_upto - w_own;
    if (share >= 0.0f) limit.weight = fmax((double)share * (double)sum_across<WAVES>(s.part64), 1.0);
    bool reached = limit.reached(n_before, w_before) || tid * OWN > stop;
#pragma unroll
    for (int b = 0; b < OWN; ++b) {
        const bool now = limit.reached(n_before + n[b], w_before + w[b]) || tid * OWN + b >= stop;
        if (now && !reached) s.bin = tid * OWN + b, s.before = n_before, s.weight_before = w_before, s.inside = n[b];  // (once at most)
        reached = now;
        n_before += n[b], w_before += w[b];
    }
    __syncthreads();
}

// found(logit, index) in one thread, for the element of piece r (first index j) at which the running sum passes target, if it is
// in this lane's piece.  own: sum of the piece; before: of all pieces before the wave's 64.
template <typename T, typename F, typename G>
__device__ __forceinline__ void find_in_piece(uint4 r, int j, u64 own, u64 before, u64 target, F value, G found) {
    const u64 upto = before + wave_scan(own);
    u64 at = upto - own;
    if (at > target || upto <= target) return;
#pragma unroll 1
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) {
        const float z = element<T>(r, e);
        const u64 v = value(z, j + e);
        if (at <= target && at + v > target) found(z, j + e);
        at += v;
    }
}

// The index of the (target + 1)th logit with that key, in s.rank.
template <int THREADS, typename T>
__device__ void find_equal(const Row<T> &row, SearchLds &s, uint32_t key, u64 target) {
    const float z_low = key_value(key);
    u64 sum = 0;
    row.each_from(z_low, [&](float z, int) { sum += order_key(z) == key; });
    sum = wave_sum(sum);
    __syncthreads();
    if (threadIdx.x == 0) s.rank = 0x7FFFFFFF;  // (if there are fewer)
    if ((threadIdx.x & 63) == 0) s.part64[threadIdx.x >> 6] = sum;
    __syncthreads();
    u64 before = sum_before<THREADS / 64>(s.part64);
    if (before <= target && before + sum > target) {
        auto is_equal = [&](float z, int) { return (u64)(order_key(z) == key); };
        for (int i = 0; i < row.rounds; ++i) {
            u64 own = 0;
            row.piece(i, [&](float z, int j) { own += is_equal(z, j); });
            const u64 all = wave_sum(own);
            if (before + all > target) {
                find_in_piece<T>(row.load(i), row.index(i), own, before, target, is_equal, [&](float, int j) { s.rank = j; });
                break;
            }
            before += all;
        }
    }
    __syncthreads();
}

// Cuts among the s.inside logits with keys low .. high, which are those in which the limit is reached, counting from s.before and
// s.weight_before.  source: gives at least these (each_from()); row: the whole row in memory.
template <int THREADS, bool BY_WEIGHT, typename R, typename T>
__device__ __forceinline__ Cut cut_among(const R &source, const Row<T> &row, const Weight &weight, SearchLds &s, Limit limit, uint32_t low, uint32_t high, int fraction) {
    constexpr int OWN = BINS / THREADS;
    auto weigh = [&](float z) { return BY_WEIGHT ? fixed_weight(weight.log2_of(z), fraction) : 0ull; };
    while (s.inside > MEMBERS) {
        const float z_low = key_value(low);
        if (low == high) {  // equal logits: as many of them as are needed, lowest indexes first
            u64 need = limit.count - s.before;
            const u64 w = weigh(z_low);
            if (BY_WEIGHT && w > 0 && limit.weight < INFINITY) {
                u64 m = (u64)fmax((limit.weight - (double)s.weight_before) / (double)w - 1.0, 1.0);
                while (m < need && !limit.reached(s.before, s.weight_before + m * w)) ++m;
                need = m < need ? m : need;
            }
            find_equal<THREADS>(row, s, low, need - 1);
            return Cut{low, s.rank};
        }
        const uint32_t spread = (high - low) / BINS;
        const int shift = spread ? 32 - __builtin_clz(spread) : 0;  // (the smallest with less than BINS intervals)
        __syncthreads();
        for (int b = threadIdx.x; b < BINS; b += THREADS) s.count[b] = 0, s.weight[b] = 0;
        __syncthreads();
        source.each_from(z_low, [&](float z, int) {
            const uint32_t k = order_key(z);
            if (k <= high) {
                atomicAdd(&s.count[(high - k) >> shift], 1u);
                if (BY_WEIGHT) atomicAdd(&s.weight[(high - k) >> shift], weigh(z));
            }
        });
        __syncthreads();
        uint32_t n[OWN];
        u64 w[OWN];
        for (int b = 0; b < OWN; ++b) n[b] = s.count[threadIdx.x * OWN + b], w[b] = s.weight[threadIdx.x * OWN + b];
        find_bin<THREADS>(s, limit, -1.0f, n, w);
        if (s.bin < 0) return Cut{low, 0x7FFFFFFF};  // (weights of a range and of its members differ by roundings: all of them)
        high -= (uint32_t)s.bin << shift;
        if ((high - low) >> shift > 0) low = high - ((1u << shift) - 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    source.each_from(key_value(low), [&](float z, int j) {
        const uint32_t k = order_key(z);
        if (k <= high) s.member[min(atomicAdd(&s.n, 1), MEMBERS - 1)] = (u64)k << 32 | (uint32_t)~j;
    });
    __syncthreads();
    if (threadIdx.x < 64) {
        const int n = min(s.n, MEMBERS);
        const u64 own = (int)threadIdx.x < n ? s.member[threadIdx.x] : 0;
        const u64 w = BY_WEIGHT && own ? weigh(key_value((uint32_t)(own >> 32))) : 0;
        uint32_t n_upto = 0;
        u64 w_upto = 0;
        for (int o = 0; o < n; ++o) {
            const bool upto = read_lane(own, o) >= own;
            n_upto += upto;
            if (BY_WEIGHT) w_upto += upto ? read_lane(w, o) : 0;
        }
        // the first that reaches the limit, or the last (weights of a range and of its members differ by roundings)
        const bool reached = own && (n_upto == (uint32_t)n || limit.reached(s.before + n_upto, s.weight_before + w_upto));
        const uint32_t rank = wave_all(reached ? n_upto : 0xFFFFFFFFu, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
        if (reached && n_upto == rank) s.member[0] = own;
        if (n == 0 && threadIdx.x == 0) s.member[0] = (u64)high << 32;  // (nothing there: what is above, and no index)
    }
    __syncthreads();
    return Cut{(uint32_t)(s.member[0] >> 32), (int)~(uint32_t)s.member[0]};
}

// The maximum of a row; NaN is none.
template <int THREADS, typename R>
__device__ float largest(const R &row, float *part) {
    float m = -INFINITY;
    row.each([&](float z, int) { m = fmaxf(m, z); });
    return block_all<THREADS>(m, part, [](float a, float b) { return fmaxf(a, b); });
}

// Rows go out in launches of fewer than 2^32 threads.
template <typename F>
hipError_t by_slices(int rows, long most, F launch) {
    for (long r = 0; r < rows; r += most) {
        launch((int)r, (int)(rows - r < most ? rows - r : most));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// f(pieces a lane holds, threads of the workgroup), as constants: the smallest workgroup that holds a row of so many pieces.
template <typename F>
hipError_t by_size(int pieces, F f) {
    using std::integral_constant;
    if (pieces <= 256) return f(integral_constant<int, 1>{}, integral_constant<int, 256>{});
    if (pieces <= 1024) return f(integral_constant<int, 4>{}, integral_constant<int, 256>{});
    if (pieces <= 4096) return f(integral_constant<int, 8>{}, integral_constant<int, 512>{});
    return f(integral_constant<int, 8>{}, integral_constant<int, 1024>{});
}

}  // namespace sushi
