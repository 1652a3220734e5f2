// Operators that pick the leading part of a row's order (logits.h): sampling and the top logits.
//
// Both need the last kept position of the order: the first one at which the number of logits reaches k or (sampling) their
// summed weight reaches top_p of the row's sum.  No row is sorted for it.  A histogram over t = log2 of the weight
// (its intervals are coarse, but in the order of the row) says in which interval the position lies; the members of that
// interval, a few dozen as a rule, are then ranked among each other, and an interval with many members is first cut
// finer by further histograms over the order key itself, until few members or one key is left.
//
// Weights are summed in 64-bit fixed point: the sums are the same in whatever order they are made (atomics in LDS), and a
// class whose interval of the sum is hit by the random number is the same in every run.  Which class that is is decided
// next to borders, so a weight has 64 bits too: 24 bits would let one draw in a few hundred rows of 100 000 logits go to
// a neighbour.
#include "logits_device.h"

namespace sushi {

namespace {

typedef unsigned long long u64;

constexpr int BINS = 1024;
constexpr double BINS_PER_LOG2 = 24.0;  // intervals of a factor 1.03, down to 2^-42 of the largest weight
constexpr int MEMBERS = 256;            // that are ranked by comparing each with each

struct SearchLds {
    uint32_t count[BINS];
    u64 weight[BINS];
    u64 w[MEMBERS];  // members of the interval that is cut no further
    uint32_t key[MEMBERS];
    int index[MEMBERS];
    u64 part64[16];
    uint32_t part32[16];
    int bin;  // what find_bin() found: the interval, what lies before it, its members
    uint32_t before, inside;
    u64 weight_before, total;
    uint32_t key_low, key_high;
    int n, rank;
};

// The last kept position of an order.
struct Cut {
    uint32_t key;
    int index;
    __device__ __forceinline__ bool keeps(uint32_t k, int j) const { return k > key || (k == key && j <= index); }
};

__device__ __forceinline__ int bin_of(double t) { return (int)fmin(fmax(t * -BINS_PER_LOG2, 0.0), BINS - 1.0); }

// A weight as a whole number of 2^-fraction (fraction <= 50), rounded: 2^52 is added, the number stands in the low bits.
__device__ __forceinline__ u64 fixed_weight(double t, int fraction) {
    return (u64)__double_as_longlong(ldexp(exp2_64<11>(t), fraction) + 4503599627370496.0) & ((1ull << 52) - 1);
}
// Bits behind the point for sums of n weights: below 2^63.
__host__ __device__ inline int fraction_bits(int n) {
    int lg = 0;
    while ((1 << lg) < n) ++lg;
    return lg > 12 ? 62 - lg : 50;
}

// When the order is cut: at the first position where this many logits, or this weight, has been reached.
struct Limit {
    uint32_t count;
    double weight;
    __device__ __forceinline__ bool reached(uint32_t n, u64 w) const { return n >= count || (double)w >= weight; }
};

// Finds the interval of the histogram in which the limit is reached, counting from (before, weight_before); s.bin = -1: in none.
// top_p >= 0: the limit's weight is that share of the histogram's whole sum.
template <int THREADS>
__device__ void find_bin(SearchLds &s, Limit &limit, float top_p) {
    constexpr int OWN = BINS / THREADS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t n0 = s.before;
    const u64 w0 = s.weight_before;
    uint32_t n = 0;
    u64 w = 0;
    for (int b = 0; b < OWN; ++b) n += s.count[tid * OWN + b], w += s.weight[tid * OWN + b];
    const uint32_t n_upto = wave_scan(n, lane);
    const u64 w_upto = wave_scan(w, lane);
    if (lane == 63) s.part32[wave] = n_upto, s.part64[wave] = w_upto;
    if (tid == 0) s.bin = -1;
    __syncthreads();
    uint32_t n_before = n0 + n_upto - n;
    u64 w_before = w0 + w_upto - w, total = 0;
    for (int v = 0; v < THREADS / 64; ++v) {
        if (v < wave) n_before += s.part32[v], w_before += s.part64[v];
        total += s.part64[v];
    }
    if (top_p >= 0.0f) limit.weight = fmax((double)top_p * (double)total, 1.0);
    if (!limit.reached(n_before, w_before) && limit.reached(n_before + n, w_before + w)) {  // (one thread at most)
        int b = tid * OWN;
        while (!limit.reached(n_before + s.count[b], w_before + s.weight[b])) n_before += s.count[b], w_before += s.weight[b], ++b;
        s.bin = b, s.before = n_before, s.weight_before = w_before, s.inside = s.count[b];
    }
    if (tid == 0) s.total = total;
    __syncthreads();
}

template <int THREADS>
__device__ __forceinline__ void clear_histogram(SearchLds &s) {
    for (int b = threadIdx.x; b < BINS; b += THREADS) s.count[b] = 0, s.weight[b] = 0;
}

// Sum of value(logit, index) over the row; wave[w]: LDS, the part of wave w.
template <int THREADS, typename R, typename F>
__device__ u64 sum_by_waves(const R &row, u64 *wave, F value) {
    u64 sum = 0;
    row.each([&](float z, int j) { sum += value(z, j); });
    sum = wave_sum(sum);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < THREADS / 64; ++w) sum += wave[w];
    return sum;
}

// found(logit, index, value), in one thread, for the first element in the order of the indexes at which the running sum of the values
// exceeds target.  wave: as sum_by_waves() left it.
template <typename R, typename F, typename G>
__device__ void first_beyond(const R &row, const u64 *wave, u64 target, F value, G found) {
    const int lane = threadIdx.x & 63, me = threadIdx.x >> 6;
    u64 before = 0;
    for (int w = 0; w < me; ++w) before += wave[w];
    if (before > target || before + wave[me] <= target) return;
    for (int i = 0; i < row.rounds; ++i) {
        u64 own = 0;
        row.piece(i, [&](float z, int j) { own += value(z, j); });
        const u64 upto = before + wave_scan(own, lane);
        const u64 all = __shfl(upto, 63);
        if (all > target) {
            u64 at = upto - own;
            if (at <= target && upto > target)
                row.piece(i, [&](float z, int j) {
                    const u64 v = value(z, j);
                    if (at <= target && at + v > target) found(z, j, v);
                    at += v;
                });
            return;
        }
        before = all;
    }
}

// The cut of a row's order at limit.  BY_WEIGHT: sums of weights are taken along (a share top_p of the row's sum is the limit where
// it is in [0, 1)); s.total is the row's sum then.  Every logit that has a weight (an ordered key) takes part.
template <int THREADS, bool BY_WEIGHT, typename R>
__device__ Cut find_cut(const R &row, const Weight &weight, SearchLds &s, uint32_t count, float top_p, int fraction) {
    Limit limit{count, INFINITY};
    clear_histogram<THREADS>(s);
    if (threadIdx.x == 0) s.before = 0, s.weight_before = 0, s.key_low = 0xFFFFFFFFu, s.key_high = 0, s.n = 0, s.rank = MEMBERS;
    __syncthreads();
    row.each([&](float z, int) {
        if (order_key(z) != KEY_NONE) {
            const double t = weight.log2_of(z);
            const int b = bin_of(t);
            atomicAdd(&s.count[b], 1u);
            if (BY_WEIGHT) atomicAdd(&s.weight[b], fixed_weight(t, fraction));
        }
    });
    __syncthreads();
    find_bin<THREADS>(s, limit, BY_WEIGHT ? top_p : -1.0f);
    if (s.bin < 0) return Cut{KEY_NONE + 1, 0x7FFFFFFF};  // (never reached: all are kept)
    const int bin = s.bin;
    uint32_t low = 0, high = 0;  // keys that are still in question, once `by_key`
    bool by_key = false;
    auto member = [&](float z, uint32_t k) {
        return by_key ? k >= low && k <= high : k != KEY_NONE && bin_of(weight.log2_of(z)) == bin;
    };
    while (s.inside > MEMBERS) {
        if (!by_key) {
            row.each([&](float z, int) {
                const uint32_t k = order_key(z);
                if (member(z, k)) atomicMin(&s.key_low, k), atomicMax(&s.key_high, k);
            });
            __syncthreads();
            low = s.key_low, high = s.key_high, by_key = true;
        }
        if (low == high) {  // equal logits: as many of them as are needed, lowest indexes first
            const u64 w = BY_WEIGHT ? fixed_weight(weight.log2_of(key_value(low)), fraction) : 0;
            u64 need = count - s.before;
            if (BY_WEIGHT && w > 0 && limit.weight < INFINITY) {
                u64 m = (u64)fmax((limit.weight - (double)s.weight_before) / (double)w - 1.0, 1.0);
                while (m < need && !limit.reached(s.before, s.weight_before + m * w)) ++m;
                need = m < need ? m : need;
            }
            auto is_member = [&](float z, int) { return (u64)(order_key(z) == low); };
            sum_by_waves<THREADS>(row, s.part64, is_member);
            first_beyond(row, s.part64, need - 1, is_member, [&](float, int j, u64) { s.rank = j; });
            __syncthreads();
            return Cut{low, s.rank};
        }
        int shift = 0;
        while ((high - low) >> shift >= (uint32_t)BINS) ++shift;
        clear_histogram<THREADS>(s);
        __syncthreads();
        row.each([&](float z, int) {
            const uint32_t k = order_key(z);
            if (member(z, k)) {
                atomicAdd(&s.count[(high - k) >> shift], 1u);
                if (BY_WEIGHT) atomicAdd(&s.weight[(high - k) >> shift], fixed_weight(weight.log2_of(z), fraction));
            }
        });
        __syncthreads();
        find_bin<THREADS>(s, limit, -1.0f);
        if (s.bin < 0) return Cut{low, 0x7FFFFFFF};  // (the members reached it before, with the same sums)
        high -= (uint32_t)s.bin << shift;
        if ((high - low) >> shift > 0) low = high - ((1u << shift) - 1);
    }
    row.each([&](float z, int j) {
        const uint32_t k = order_key(z);
        if (member(z, k)) {
            const int at = min(atomicAdd(&s.n, 1), MEMBERS - 1);
            s.key[at] = k, s.index[at] = j;
            if (BY_WEIGHT) s.w[at] = fixed_weight(weight.log2_of(z), fraction);
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
        if (limit.reached(s.before + upto, s.weight_before + w)) atomicMin(&s.rank, (int)upto - 1);
        s.count[i] = upto - 1;  // (the histogram is done with)
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS)
        if ((int)s.count[i] == s.rank) s.bin = i;
    __syncthreads();
    return Cut{s.key[s.bin], s.index[s.bin]};
}

template <int THREADS, typename R>
__device__ uint32_t largest_key(const R &row, uint32_t *part) {
    uint32_t k = 0;
    row.each([&](float z, int) { k = max(k, order_key(z)); });
    return block_all<THREADS>(k, part, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a, int row0) {
    __shared__ SearchLds s;
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Row<T> row(a.in, r, wave, THREADS / 64, lane);
    const uint32_t best = largest_key<THREADS>(row, s.part32);
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if (best <= KEY_NONE) {  // nothing to draw from
        if (threadIdx.x == 0) {
            a.classes[r] = -1;
            if (a.log_prob) a.log_prob[r] = -INFINITY;
        }
        return;
    }
    if (!(temperature > 0.0f)) {  // the first of the order
        __syncthreads();
        int j = 0x7FFFFFFF;
        row.each([&](float z, int at) { j = min(j, order_key(z) == best ? at : 0x7FFFFFFF); });
        j = block_all<THREADS>(j, reinterpret_cast<int *>(s.part32), [](int p, int q) { return p < q ? p : q; });
        if (threadIdx.x == 0) {
            a.classes[r] = j;
            if (a.log_prob) a.log_prob[r] = 0.0f;
        }
        return;
    }
    const Weight weight(key_value(best), 1.0 / (double)temperature);
    const int fraction = fraction_bits(a.in.n);
    const int k = a.top_k && a.top_k[r] > 0 ? min(a.top_k[r], a.in.n) : a.in.n;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f;
    const float min_p = a.min_p ? fminf(fmaxf(a.min_p[r], 0.0f), 1.0f) : 0.0f;
    const double t_min = min_p > 0.0f ? log2((double)min_p) : -INFINITY;
    Cut cut{KEY_NONE + 1, 0x7FFFFFFF};
    if (top_p < 1.0f)
        cut = find_cut<THREADS, true>(row, weight, s, k, fmaxf(top_p, 0.0f), fraction);
    else if (k < a.in.n)
        cut = find_cut<THREADS, false>(row, weight, s, k, -1.0f, fraction);
    auto kept = [&](float z, int j) {
        const double t = weight.log2_of(z);
        return cut.keeps(order_key(z), j) && t >= t_min ? fixed_weight(t, fraction) : 0;
    };
    const u64 total = sum_by_waves<THREADS>(row, s.part64, kept);
    const double u = fminf(fmaxf(a.uniform[r], 0.0f), 1.0f - 5.9604645e-08f);  // (into [0, 1); NaN: 0)
    const u64 target = min((u64)(u * (double)total), total - 1);
    first_beyond(row, s.part64, target, kept, [&](float z, int j, u64) {
        a.classes[r] = j;
        if (a.log_prob) a.log_prob[r] = (float)((weight.log2_of(z) + fraction - log2((double)total)) * 6.931471805599453094e-01);
    });
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void top_logits_kernel(TopArgs a, int row0) {
    __shared__ SearchLds s;
    __shared__ u64 order[LOGITS_MAX_TOP];
    __shared__ int n_kept;
    __shared__ double part[2][THREADS / 64];
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Row<T> row(a.in, r, wave, THREADS / 64, lane);
    const uint32_t best = largest_key<THREADS>(row, s.part32);
    const Weight weight(key_value(best), 1.0 / (double)a.temperature);
    Cut cut{KEY_NONE + 1, 0x7FFFFFFF};
    if (best > KEY_NONE && a.k < a.in.n) cut = find_cut<THREADS, false>(row, weight, s, a.k, -1.0f, 0);
    // the kept ones, sorted in LDS (keys above inverted indexes; zeros, smaller than any, fill up to a power of two)
    int size = 1;
    while (size < a.k) size *= 2;
    if (threadIdx.x == 0) n_kept = 0;
    for (int i = threadIdx.x; i < size; i += THREADS) order[i] = 0;
    __syncthreads();
    double inside = 0.0, outside = 0.0;
    row.each([&](float z, int j) {
        const uint32_t k = order_key(z);
        const bool keep = k != KEY_NONE && cut.keeps(k, j);
        if (keep) order[min(atomicAdd(&n_kept, 1), LOGITS_MAX_TOP - 1)] = (u64)k << 32 | (uint32_t)~j;
        const double w = exp2_64<7>(weight.log2_of(z));
        inside += keep ? w : 0.0;
        outside += keep ? 0.0 : w;
    });
    inside = block_sum<THREADS>(inside, part[0]);
    outside = block_sum<THREADS>(outside, part[1]);
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
    for (int i = threadIdx.x; i < a.k; i += THREADS) {
        a.values[r * a.k + i] = order[i] ? key_value((uint32_t)(order[i] >> 32)) : -INFINITY;
        a.classes[r * a.k + i] = order[i] ? (int)~(uint32_t)order[i] : -1;
    }
    if (threadIdx.x == 0 && a.rest) a.rest[r] = best > KEY_NONE ? (float)(outside / (inside + outside)) : 0.0f;
}

constexpr int THREADS = 256;

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

}  // namespace

hipError_t launch_sample(const SampleArgs &a, void *, hipStream_t s) {
    return by_slices(a.in.rows, THREADS, [&](int r, int n) {
        if (a.in.bf16)
            sample_kernel<uint16_t, THREADS><<<n, THREADS, 0, s>>>(a, r);
        else
            sample_kernel<float, THREADS><<<n, THREADS, 0, s>>>(a, r);
    });
}

hipError_t launch_top_logits(const TopArgs &a, void *, hipStream_t s) {
    return by_slices(a.in.rows, THREADS, [&](int r, int n) {
        if (a.in.bf16)
            top_logits_kernel<uint16_t, THREADS><<<n, THREADS, 0, s>>>(a, r);
        else
            top_logits_kernel<float, THREADS><<<n, THREADS, 0, s>>>(a, r);
    });
}

}  // namespace sushi
