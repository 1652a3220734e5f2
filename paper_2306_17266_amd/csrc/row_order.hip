// Operators that pick the leading part of a row's order (logits.h): sampling and the top logits.
//
// Both need the last kept position of the order: the first one at which the number of logits reaches k or (sampling) their
// summed weight reaches top_p of the row's sum.  No row is sorted for it.  A histogram over a grid on the logits, 12 intervals for
// each factor 2 of the weight, says in which interval the position lies; the members of that interval, a few dozen as a
// rule, are then ranked among each other, and an interval with many members is first cut finer by further histograms
// over the order key itself, until few members or one key is left.
//
// Sums of weights are whole numbers (fixed point in 64 bits): the same in whatever order atomics in LDS make them, so that a class
// whose interval of the sum is hit by the random number is the same in every run.  Which class that is is decided next to borders,
// so a weight has more than 32 bits: 24 would let one draw in a few hundred rows of 100 000 logits go to a neighbour.
#include "logits_device.h"

namespace sushi {

namespace {

typedef unsigned long long u64;

constexpr int BINS = 1024;
constexpr double BINS_PER_LOG2 = 12.0;  // 1024: down to 2^-85 of the largest weight, the rest in the last one
constexpr double LN2 = 6.931471805599453094e-01;
constexpr int MEMBERS = 256;            // that are ranked by comparing each with each
constexpr int TOP_LIST = 2 * LOGITS_MAX_TOP;

struct SearchLds {
    u64 weight[BINS + 1];  // (the last: of what is in no order)
    uint32_t count[BINS];
    u64 w[MEMBERS];  // members of the interval that is cut no further
    uint32_t key[MEMBERS];
    int index[MEMBERS];
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
__host__ __device__ inline int bits_of(int n) {  // n <= 2^bits_of(n)
    int lg = 0;
    while ((1 << lg) < n) ++lg;
    return lg;
}
// Bits behind the point for sums of n weights: below 2^63.
__device__ __forceinline__ int fraction_bits(int n) { return min(62 - bits_of(n), 50); }

// The grid: a logit lies in interval floor(place), counted downwards from the largest logit, whose place is 0.  (A row of equal
// logits has exact sums that way, and its cut is where the count says.)
struct Grid {
    double best, scale;
    __device__ __forceinline__ Grid(float m, double inv_t) : best(m), scale(inv_t * (1.4426950408889634074 * BINS_PER_LOG2)) {}
    // (rounded by itself: fused with a subtraction it would be another number in each use)
    __device__ __forceinline__ double place(float z) const {
#pragma clang fp contract(off)
        return (best - (double)z) * scale;
    }
    // Key of the smallest logit in intervals 0 .. b.
    __device__ uint32_t lowest_key(int b) const {
        const uint32_t lowest = KEY_NONE + 1, highest = order_key((float)best);
        const double x = b + 1.0;
        if (b >= BINS - 1 || !(scale > 0.0)) return lowest;
        uint32_t k = order_key((float)fmin(fmax(best - x / scale, -3.4028234663852886e38), 3.4028234663852886e38));
        while (k > lowest && place(key_value(k - 1)) < x) --k;
        while (k < highest && place(key_value(k)) >= x) ++k;
        return k;
    }
};

// An interval of the grid's histogram in one word: how many, above the sum of what their weights lack of the interval's upper end
// (relative to it, 1 - 2^(-1/12) = 0.056 at most), in fixed point.
struct Packed {
    int fraction, count_at;
    double c[6];  // of the power series of 1 - 2^(-x / 12), what is left out 2e-11 at most, as fixed point
    u64 one_more;
    __device__ __forceinline__ Packed(int n) : fraction(min(40, 66 - 2 * bits_of(n))), count_at(fraction - 4 + bits_of(n)) {
        constexpr double x = LN2 / BINS_PER_LOG2;
        const double unit = ldexp(1.0, fraction);
        c[0] = x * unit, c[1] = -x * x / 2 * unit, c[2] = x * x * x / 6 * unit, c[3] = -x * x * x * x / 24 * unit;
        c[4] = x * x * x * x * x / 120 * unit, c[5] = -x * x * x * x * x * x / 720 * unit;
        one_more = (1ull << count_at) - 0x4330000000000000ull;  // (less the bits of 2^52)
    }
    __device__ __forceinline__ u64 one(double below) const {  // below: place - floor(place)
        double p = fma(c[5], below, c[4]);
        p = fma(p, below, c[3]), p = fma(p, below, c[2]), p = fma(p, below, c[1]), p = fma(p, below, c[0]);
        return (u64)__double_as_longlong(fma(p, below, 4503599627370496.0)) + one_more;
    }
    __device__ __forceinline__ uint32_t count(u64 v) const { return (uint32_t)(v >> count_at); }
    // Weight of interval b, relative to the largest logit's.
    __device__ __forceinline__ double weight(u64 v, int b) const {
        const double lack = ldexp((double)(v & ((1ull << count_at) - 1)), -fraction);
        return ((double)count(v) - lack) * exp2_64<11>(b * (-1.0 / BINS_PER_LOG2));
    }
};

// When the order is cut: at the first position where this many logits, or this weight, has been reached.
struct Limit {
    uint32_t count;
    double weight;
    __device__ __forceinline__ bool reached(uint32_t n, u64 w) const { return n >= count || (double)w >= weight; }
};

// Finds the interval in which the limit is reached, counting from (s.before, s.weight_before); s.bin = -1: in none.  n, w: this
// thread's run of intervals, their members and weights.  Returns the sum of all weights; share >= 0: that share of it is the limit's weight.
template <int THREADS>
__device__ u64 find_bin(SearchLds &s, Limit &limit, float share, const uint32_t (&n)[BINS / THREADS], const u64 (&w)[BINS / THREADS]) {
    constexpr int OWN = BINS / THREADS;
    const int tid = threadIdx.x, wave = tid >> 6;
    uint32_t n_before = s.before, n_own = 0;
    u64 w_before = s.weight_before, w_own = 0, total = 0;
#pragma unroll
    for (int b = 0; b < OWN; ++b) n_own += n[b], w_own += w[b];
    const uint32_t n_upto = wave_scan(n_own);
    const u64 w_upto = wave_scan(w_own);
    if ((tid & 63) == 63) s.part32[wave] = n_upto, s.part64[wave] = w_upto;
    if (tid == 0) s.bin = -1;
    __syncthreads();
    total = sum_across<THREADS / 64>(s.part64);
    n_before += sum_before<THREADS / 64>(s.part32) + n_upto - n_own;
    w_before += sum_before<THREADS / 64>(s.part64) + w_upto - w_own;
    if (share >= 0.0f) limit.weight = fmax((double)share * (double)total, 1.0);
    if (!limit.reached(n_before, w_before) && limit.reached(n_before + n_own, w_before + w_own)) {  // (one thread at most)
        bool found = false;
#pragma unroll
        for (int b = 0; b < OWN; ++b) {
            if (!found && limit.reached(n_before + n[b], w_before + w[b])) {
                found = true;
                s.bin = tid * OWN + b, s.before = n_before, s.weight_before = w_before, s.inside = n[b];
            }
            n_before += n[b], w_before += w[b];
        }
    }
    __syncthreads();
    return total;
}

template <int THREADS>
__device__ __forceinline__ void clear_histogram(SearchLds &s) {
    for (int b = threadIdx.x; b < BINS; b += THREADS) s.count[b] = 0, s.weight[b] = 0;
}

// Sums of value(logit, index) by pieces (HeldRow) and over the row; wave[w]: LDS, the part of wave w.  Only what is at least
// z_low has a value; FEW: which is not much of the row.
template <int THREADS, bool FEW, typename T, int N, typename F>
__device__ u64 sum_values(const HeldRow<T, N> &row, u64 (&own)[N], u64 *wave, float z_low, F value) {
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        own[i] = 0;
        if (i < row.rounds) {
            const int j = row.index(i);
            if (FEW) {
                from_piece<T>(row.raw[i], j, z_low, [&](float z, int at) { own[i] += value(z, at); });
            } else {
                float v[HeldRow<T, N>::PER];
                unpack<T>(row.raw[i], v);
#pragma unroll
                for (int e = 0; e < HeldRow<T, N>::PER; ++e) own[i] += value(v[e], j + e);
            }
        }
        sum += own[i];
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    return sum_across<THREADS / 64>(wave);
}
template <int THREADS, bool FEW, typename T, int N, typename F>
__device__ u64 sum_values(const Row<T> &row, u64 (&)[N], u64 *wave, float z_low, F value) {
    u64 sum = 0;
    row.each_from(z_low, [&](float z, int j) { sum += value(z, j); });
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    return sum_across<THREADS / 64>(wave);
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

// found(logit, index), in one thread, for the first element in the order of the indexes at which the running sum of the values
// exceeds target.  own, wave: as sum_values() left them.
template <int THREADS, typename T, int N, typename F, typename G>
__device__ void first_beyond(const HeldRow<T, N> &row, const u64 (&own)[N], const u64 *wave, u64 target, F value, G found) {
    u64 before = sum_before<THREADS / 64>(wave);
    if (before > target || before + wave[threadIdx.x >> 6] <= target) return;
    uint4 r = row.raw[0];
    u64 sum = own[0];
    int at = 0;
    bool passed = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const u64 all = wave_sum(own[i]);
        r = choose(passed, r, row.raw[i]), sum = passed ? sum : own[i], at = passed ? at : i;
        passed |= before + all > target;
        before += passed ? 0 : all;
    }
    find_in_piece<T>(r, row.index(at), sum, before, target, value, found);
}
template <int THREADS, typename T, int N, typename F, typename G>
__device__ void first_beyond(const Row<T> &row, const u64 (&)[N], const u64 *wave, u64 target, F value, G found) {
    u64 before = sum_before<THREADS / 64>(wave);
    if (before > target || before + wave[threadIdx.x >> 6] <= target) return;
    for (int i = 0; i < row.rounds; ++i) {
        u64 own = 0;
        row.piece(i, [&](float z, int j) { own += value(z, j); });
        const u64 all = wave_sum(own);
        if (before + all > target) {
            find_in_piece<T>(row.load(i), row.index(i), own, before, target, value, found);
            return;
        }
        before += all;
    }
}

// Cuts on among the s.inside logits with keys low .. high, which are those in which the limit is reached, counting from s.before and
// s.weight_before.  R: any source of logits with each_from().
template <int THREADS, bool BY_WEIGHT, int N, typename R>
__device__ __forceinline__ Cut cut_among(const R &row, const Weight &weight, SearchLds &s, const Limit limit_, uint32_t low, uint32_t high, int fraction) {
    constexpr int OWN = BINS / THREADS;
    Limit limit = limit_;
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
            if (need > s.inside) need = s.inside;
            auto is_member = [&](float z, int) { return (u64)(order_key(z) == low); };
            u64 own[N];
            __syncthreads();
            sum_values<THREADS, true>(row, own, s.part64, z_low, is_member);
            first_beyond<THREADS>(row, own, s.part64, need - 1, is_member, [&](float, int j) { s.rank = j; });
            __syncthreads();
            return Cut{low, s.rank};
        }
        int shift = 0;
        while ((high - low) >> shift >= (uint32_t)BINS) ++shift;
        __syncthreads();
        clear_histogram<THREADS>(s);
        __syncthreads();
        row.each_from(z_low, [&](float z, int) {
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
        if (s.bin < 0) return Cut{low, 0x7FFFFFFF};  // (weights of a grid's interval and of its members differ by roundings: all of them)
        high -= (uint32_t)s.bin << shift;
        if ((high - low) >> shift > 0) low = high - ((1u << shift) - 1);
    }
    if (threadIdx.x == 0) s.n = 0, s.rank = MEMBERS;
    __syncthreads();
    row.each_from(key_value(low), [&](float z, int j) {
        const uint32_t k = order_key(z);
        if (k <= high) {
            const int at = min(atomicAdd(&s.n, 1), MEMBERS - 1);
            s.key[at] = k, s.index[at] = j;
            if (BY_WEIGHT) s.w[at] = weigh(z);
        }
    });
    __syncthreads();
    const int n = min(s.n, MEMBERS);
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint32_t k = s.key[i];
        const int j = s.index[i];
        uint32_t upto = 0;
        u64 w = 0;
        for (int o = 0; o < n; ++o)
            if (s.key[o] > k || (s.key[o] == k && s.index[o] <= j)) {
                ++upto;
                if (BY_WEIGHT) w += s.w[o];
            }
        s.count[i] = upto - 1;  // (the histogram is done with)
        if ((int)upto == n || limit.reached(s.before + upto, s.weight_before + w)) atomicMin(&s.rank, (int)upto - 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS)
        if ((int)s.count[i] == s.rank) s.bin = i;
    __syncthreads();
    return Cut{s.key[s.bin], s.index[s.bin]};
}

// What a histogram over the grid says of a row.
struct Found {
    uint32_t low, high;  // keys of the interval in which the limit is reached; low > high: in none
    double below;        // SUMS: weight of the intervals behind it
    double total;        // SUMS: of the row
};

// BY_WEIGHT: the limit has a weight, the share of the row's sum where share >= 0.  SUMS: the sums of Found (with what is
// below the grid).  For rows with a finite maximum.
template <int THREADS, bool BY_WEIGHT, bool SUMS, typename R>
__device__ Found search_grid(const R &row, const Weight &weight, const Grid &grid, SearchLds &s, double *part_d, Limit &limit, float share, int n,
                             int fraction) {
    constexpr int OWN = BINS / THREADS;
    const Packed packed(n);
    for (int b = threadIdx.x; b < BINS; b += THREADS) s.weight[b] = 0;
    if (threadIdx.x == 0) s.before = 0, s.weight_before = 0;
    __syncthreads();
    row.each([&](float z, int) {
        const double t = grid.place(z), g = floor(t);
        const int b = min((int)g, BINS - 1);
        atomicAdd(&s.weight[z > -INFINITY ? b : BINS], packed.one(t - g));  // (no branch: it would be one for each logit)
    });
    __syncthreads();
    uint32_t count[OWN];
    u64 w[OWN];
    double wd[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int b = threadIdx.x * OWN + i;
        const u64 v = s.weight[b];
        count[i] = packed.count(v), w[i] = 0, wd[i] = 0.0;
        if (b < BINS - 1 && v) {
            wd[i] = packed.weight(v, b);
            if (BY_WEIGHT) w[i] = (u64)ldexp(wd[i], fraction);
        }
    }
    find_bin<THREADS>(s, limit, share, count, w);
    Found f{1, 0, 0.0, 0.0};
    const int bin = s.bin;
    if (bin >= 0) f.low = grid.lowest_key(bin), f.high = bin > 0 ? grid.lowest_key(bin - 1) - 1 : 0xFFFFFFFFu;
    if (SUMS) {
        double tail = 0.0;
        if (packed.count(s.weight[BINS - 1])) {
            const uint32_t last = grid.lowest_key(BINS - 2);
            row.each([&](float z, int) {
                if (order_key(z) < last) tail += exp2_64<6>(weight.log2_of(z));
            });
        }
        double below = 0.0, total = tail;
#pragma unroll
        for (int i = 0; i < OWN; ++i) total += wd[i], below += bin >= 0 && threadIdx.x * OWN + i > bin ? wd[i] : 0.0;
        if (bin >= 0 && bin < BINS - 1) below += tail;
        f.below = block_sum<THREADS>(below, part_d);
        f.total = block_sum<THREADS>(total, part_d + 16);
    }
    return f;
}

template <int THREADS, typename R>
__device__ float largest(const R &row, float *part) {
    float m = -INFINITY;
    row.each([&](float z, int) { m = fmaxf(m, z); });
    return block_all<THREADS>(m, part, [](float a, float b) { return fmaxf(a, b); });
}

template <typename T, int N>
using Source = std::conditional_t<N == 0, Row<T>, HeldRow<T, N ? N : 1>>;

template <typename T, int N, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void sample_kernel(SampleArgs a, int row0) {
    __shared__ SearchLds s;
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Source<T, N> row(a.in, r, wave, THREADS / 64, lane);
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    const int k = a.top_k && a.top_k[r] > 0 ? min(a.top_k[r], a.in.n) : a.in.n;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f;
    const float min_p = a.min_p ? fminf(fmaxf(a.min_p[r], 0.0f), 1.0f) : 0.0f;
    const float uniform = a.uniform[r];
    float best = largest<THREADS>(row, s.part_f);
    if (best == -INFINITY) {  // nothing to draw from
        if (threadIdx.x == 0) {
            a.classes[r] = -1;
            if (a.log_prob) a.log_prob[r] = -INFINITY;
        }
        return;
    }
    if (!(temperature > 0.0f)) {  // the first of the order
        int j = 0x7FFFFFFF;
        row.each([&](float z, int at) { j = min(j, z == best ? at : 0x7FFFFFFF); });
        j = block_all<THREADS>(j, reinterpret_cast<int *>(s.part32), [](int p, int q) { return p < q ? p : q; });
        if (threadIdx.x == 0) {
            a.classes[r] = j;
            if (a.log_prob) a.log_prob[r] = 0.0f;
        }
        return;
    }
    const double inv_t = 1.0 / (double)temperature;
    if (best == INFINITY) row.only_infinite(), best = 0.0f;
    const Weight weight(best, inv_t);
    const int fraction = fraction_bits(a.in.n);
    const double t_min = min_p > 0.0f ? log2((double)min_p) : -INFINITY;
    const bool by_weight = top_p < 1.0f;
    Cut cut = keep_all();
    if (by_weight || k < a.in.n) {
        Limit limit{(uint32_t)k, INFINITY};
        const Found f = search_grid<THREADS, true, false>(row, weight, Grid(best, inv_t), s, nullptr, limit, by_weight ? fmaxf(top_p, 0.0f) : -1.0f, a.in.n, fraction);
        if (f.low <= f.high) cut = cut_among<THREADS, true, N ? N : 1>(row, weight, s, limit, f.low, f.high, fraction);
    }
    auto kept = [&](float z, int j) {
        const double t = weight.log2_of(z);
        return cut.keeps(order_key(z), j) && t >= t_min ? fixed_weight(t, fraction) : 0;
    };
    // (a first screening of what min_p leaves, a little below its border)
    double z_min = weight.best + t_min / weight.scale;
    z_min -= fabs(z_min) * 1e-6;
    const float z_low = fmaxf(key_value(cut.key), z_min > -3e38 && z_min < 3e38 ? (float)z_min : -INFINITY);
    u64 own[N ? N : 1];
    const bool few = by_weight || k < a.in.n || min_p > 0.0f;
    const u64 total = few ? sum_values<THREADS, true>(row, own, s.part64, z_low, kept)
                          : sum_values<THREADS, false>(row, own, s.part64, -INFINITY, [&](float z, int) { return fixed_weight(weight.log2_of(z), fraction); });
    const double u = fminf(fmaxf(uniform, 0.0f), 1.0f - 5.9604645e-08f);  // (into [0, 1); NaN: 0)
    const u64 target = min((u64)(u * (double)total), total - 1);
    first_beyond<THREADS>(row, own, s.part64, target, kept, [&](float z, int j) {
        a.classes[r] = j;
        if (a.log_prob) a.log_prob[r] = (float)((weight.log2_of(z) + fraction - log2((double)total)) * LN2);
    });
}

template <typename T, int N, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void top_logits_kernel(TopArgs a, int row0) {
    __shared__ SearchLds s;
    __shared__ u64 order[TOP_LIST];
    __shared__ int n_listed;
    __shared__ double part[3][16];
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Source<T, N> row(a.in, r, wave, THREADS / 64, lane);
    const float best = largest<THREADS>(row, s.part_f);
    const double inv_t = 1.0 / (double)a.temperature;
    const bool infinite = best == INFINITY;
    const Weight weight(infinite ? 0.0f : best, inv_t);
    Limit limit{(uint32_t)a.k, INFINITY};
    Found f{1, 0, 0.0, 1.0};
    if (infinite) {  // (the grid ends there: cut by keys alone)
        uint32_t ordered = 0, infinities = 0;
        row.each([&](float z, int) { ordered += z > -INFINITY, infinities += z == INFINITY; });
        ordered = block_sum<THREADS>(ordered, s.part32);
        infinities = block_sum<THREADS>(infinities, reinterpret_cast<uint32_t *>(s.part64));
        if (threadIdx.x == 0) s.before = 0, s.weight_before = 0, s.inside = ordered;
        __syncthreads();
        f.total = infinities;
        if ((int)ordered >= a.k) f.low = KEY_NONE + 1, f.high = 0xFFFFFFFFu;
    } else if (best > -INFINITY) f = search_grid<THREADS, false, true>(row, weight, Grid(best, inv_t), s, part[0], limit, -1.0f, a.in.n, 0);
    // everything down to the interval of the k-th, or, if that holds too much, down to the k-th itself
    Cut cut = keep_all();
    const bool all = f.low <= f.high && s.before + s.inside <= TOP_LIST;
    if (all)
        cut.key = f.low;
    else if (f.low <= f.high)
        cut = cut_among<THREADS, false, N ? N : 1>(row, weight, s, limit, f.low, f.high, 0);
    if (threadIdx.x == 0) n_listed = 0;
    __syncthreads();
    double outside = 0.0;  // of the interval
    row.each_from(key_value(min(cut.key, max(f.low, KEY_NONE + 1))), [&](float z, int j) {
        const uint32_t k = order_key(z);
        if (cut.keeps(k, j))
            order[min(atomicAdd(&n_listed, 1), TOP_LIST - 1)] = (u64)k << 32 | (uint32_t)~j;
        else if (k <= f.high)
            outside += exp2_64<6>(weight.log2_of(infinite ? as_infinite(z) : z));
    });
    __syncthreads();
    // sorted in LDS: keys above inverted indexes
    const int n = min(n_listed, TOP_LIST);
    int size = 1;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += THREADS) order[i] = 0;
    __syncthreads();
    for (int width = 2; width <= size; width *= 2)
        for (int d = width / 2; d > 0; d /= 2) {
            for (int i = threadIdx.x; i < size / 2; i += THREADS) {
                const int lo = (i / d) * 2 * d + i % d, hi = lo + d;
                const u64 p = order[lo], q = order[hi];
                if ((p < q) == ((lo & width) == 0)) order[lo] = q, order[hi] = p;
            }
            __syncthreads();
        }
    for (int i = threadIdx.x; i < max(n, a.k); i += THREADS) {
        const u64 v = i < n ? order[i] : 0;
        if (i < a.k) {
            a.values[r * a.k + i] = v ? key_value((uint32_t)(v >> 32)) : -INFINITY;
            a.classes[r * a.k + i] = v ? (int)~(uint32_t)v : -1;
        } else {
            const float z = key_value((uint32_t)(v >> 32));
            outside += exp2_64<6>(weight.log2_of(infinite ? as_infinite(z) : z));
        }
    }
    outside = block_sum<THREADS>(outside, part[2]);
    if (threadIdx.x == 0 && a.rest) a.rest[r] = (float)((f.below + outside) / f.total);
}

// Rows go out in launches of fewer than 2^32 threads.
template <typename F>
hipError_t by_slices(int rows, int threads, F launch) {
    const long most = (1l << 31) / threads;
    for (long r = 0; r < rows; r += most) {
        launch((int)r, (int)(rows - r < most ? rows - r : most));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// f(pieces a lane holds, threads of the workgroup) for rows of n logits, as constants: the smallest that holds a row; 0 pieces:
// the row is read again for every pass.
template <typename T, typename F>
hipError_t by_size(int n, F f) {
    const int pieces = (n + 2 * (16 / (int)sizeof(T)) - 2) / (16 / (int)sizeof(T));  // (a row may start inside its first piece)
    using std::integral_constant;
    if (pieces <= 256) return f(integral_constant<int, 1>{}, integral_constant<int, 256>{});
    if (pieces <= 1024) return f(integral_constant<int, 4>{}, integral_constant<int, 256>{});
    if (pieces <= 4096) return f(integral_constant<int, 8>{}, integral_constant<int, 512>{});
    if (pieces <= 8192) return f(integral_constant<int, 8>{}, integral_constant<int, 1024>{});
    return f(integral_constant<int, 0>{}, integral_constant<int, 1024>{});
}

template <typename T>
hipError_t sample(const SampleArgs &a, hipStream_t s) {
    return by_size<T>(a.in.n, [&](auto N, auto THREADS) {
        return by_slices(a.in.rows, THREADS, [&](int r, int n) { sample_kernel<T, decltype(N)::value, decltype(THREADS)::value><<<n, (int)THREADS, 0, s>>>(a, r); });
    });
}
template <typename T>
hipError_t top_logits(const TopArgs &a, hipStream_t s) {
    return by_size<T>(a.in.n, [&](auto N, auto THREADS) {
        return by_slices(a.in.rows, THREADS, [&](int r, int n) { top_logits_kernel<T, decltype(N)::value, decltype(THREADS)::value><<<n, (int)THREADS, 0, s>>>(a, r); });
    });
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, void *, hipStream_t s) { return a.in.bf16 ? sample<uint16_t>(a, s) : sample<float>(a, s); }
hipError_t launch_top_logits(const TopArgs &a, void *, hipStream_t s) { return a.in.bf16 ? top_logits<uint16_t>(a, s) : top_logits<float>(a, s); }

}  // namespace sushi
