// One class per row from given random numbers, under temperature, top-k, top-p and min-p (logits.h).
//
// The position at which top-k and top-p cut the order is searched with a histogram over a grid on the logits, 12 intervals for each
// factor 2 of the weight (logit_grid.h), and then among the members of one interval (row_order.h).  The answer is found in the order of the
// indexes: sums of the kept weights by waves and pieces, then the piece in which the running sum passes u times the whole.
#include "row_order.h"

namespace sushi {

namespace {

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
    __device__ __forceinline__ u64 lack(u64 v) const { return v & ((1ull << count_at) - 1); }
    // Weight of an interval's members, relative to its upper end.
    __device__ __forceinline__ double sum(uint32_t count, u64 lacking) const { return (double)count - ldexp((double)lacking, -fraction); }
};

// The histogram of what a source holds, in s.weight.
template <int THREADS, typename R>
__device__ void build_histogram(const R &row, const Grid &grid, const Packed &packed, SearchLds &s) {
    for (int b = threadIdx.x; b < BINS; b += THREADS) s.weight[b] = 0;
    __syncthreads();
    row.each([&](float z, int) {
        const double t = grid.place(z), g = floor(t);
        const int b = min((int)(g - grid.top), BINS - 1);
        atomicAdd(&s.weight[z > -INFINITY ? b : BINS], packed.one(t - g));  // (no branch: it would be one for each logit)
    });
    __syncthreads();
}

// How a row is drawn from.
struct Draw {
    float temperature, top_p, min_p, u;
    int k;
    bool first;  // the first of the order, whatever else is asked for
    __device__ __forceinline__ Draw(const SampleArgs &a, long r) {
        // (all loaded, from some row of numbers or other, before one is looked at: a branch for each would wait for each)
        const float *any = a.uniform;
        u = any[r];
        temperature = (a.temperature ? a.temperature : any)[r];
        k = (a.top_k ? a.top_k : reinterpret_cast<const int32_t *>(any))[r];
        top_p = (a.top_p ? a.top_p : any)[r];
        min_p = (a.min_p ? a.min_p : any)[r];
        u = fminf(fmaxf(u, 0.0f), 1.0f - 5.9604645e-08f);  // (into [0, 1); NaN: 0)
        temperature = a.temperature ? temperature : 1.0f;
        k = a.top_k && k > 0 ? min(k, a.in.n) : a.in.n;
        top_p = a.top_p ? top_p : 1.0f;
        min_p = a.min_p ? fminf(fmaxf(min_p, 0.0f), 1.0f) : 0.0f;
        first = !(temperature > 0.0f);
        if (first) temperature = 1.0f, k = 1, top_p = 1.0f, min_p = 0.0f;
    }
    __device__ __forceinline__ bool cuts(int n) const { return k < n || top_p < 1.0f || min_p > 0.0f; }
    __device__ __forceinline__ float share() const { return top_p < 1.0f ? fmaxf(top_p, 0.0f) : -1.0f; }
    __device__ __forceinline__ double t_min() const { return min_p > 0.0f ? log2_64((double)min_p) : -INFINITY; }
};

// Where a row is cut: interval `start` of the grid (none: BINS), and the keys in question.  All above them are kept, none below.
struct Range {
    int start;
    uint32_t low, high;
};
// count, lacking: this thread's run of intervals.  equal: members of the first that equal the maximum and are in neither.  t_min: log2
// of the weight from which min_p keeps.  s.before, s.weight_before: zero.
template <int THREADS>
__device__ Range search(SearchLds &s, const Grid &grid, const Packed &packed, float best, Limit &limit, const Draw &draw, double t_min, uint32_t (&count)[BINS / THREADS],
                        const u64 (&lacking)[BINS / THREADS], uint32_t equal, int fraction) {
    constexpr int OWN = BINS / THREADS;
    const double above = grid.place(best) - grid.top;  // of the maximum within its interval
    u64 w[OWN];
    double edge = exp2_64<11>((above - (int)threadIdx.x * OWN) * (1.0 / BINS_PER_LOG2));  // weight of an interval's upper end
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int b = threadIdx.x * OWN + i;
        double wd = b < BINS - 1 ? packed.sum(count[i], lacking[i]) * edge : 0.0;
        edge *= 9.438743126816934966e-01;  // 2^(-1/12)
        if (b == 0) count[i] += equal, wd += equal;
        w[i] = (u64)ldexp(wd, fraction);
    }
    // the interval of min_p's border; the next one too where the border lies next to it
    const double border = above - t_min * BINS_PER_LOG2;
    const int stop = (int)fmin(fmax(border - 1e-6, 0.0), (double)BINS), stop_end = (int)fmin(border + 1e-6, (double)BINS);
    find_bin<THREADS>(s, limit, draw.share(), count, w, stop);
    const int bin = s.bin;
    if (bin < 0) return Range{BINS, 1, 0};
    const int end = bin == stop ? max(stop_end, bin) : bin;
    const double unit = (double)draw.temperature * (LN2 / BINS_PER_LOG2);
    // (the lower and the upper end, in neighbouring lanes)
    const uint32_t k = lowest_key(grid, threadIdx.x & 1 ? bin - 1 : end, best, unit);
    const uint32_t low = read_lane(k, 0), above_high = read_lane(k, 1);
    if (end != bin && threadIdx.x == 0) s.inside = 0x7FFFFFFF;  // (more than is known)
    __syncthreads();
    return Range{bin, low, bin > 0 ? above_high - 1 : 0xFFFFFFFFu};
}

// Which logits are kept, and their weights.
struct Kept {
    Weight weight;
    Cut cut;
    double t_min;
    int fraction;
    __device__ __forceinline__ u64 operator()(float z, int j) const {
        const double t = weight.log2_of(z);
        return cut.keeps(order_key(z), j) && t >= t_min ? fixed_weight(t, fraction) : 0;
    }
};

__device__ __forceinline__ u64 target_of(float u, u64 total) { return min((u64)((double)u * (double)total), total - 1); }

__device__ __forceinline__ void write_answer(const SampleArgs &a, long r, int j, double log2_of, int fraction, u64 total) {
    a.classes[r] = j;
    if (a.log_prob) a.log_prob[r] = (float)((log2_of + fraction - log2_64((double)total)) * LN2);
}
__device__ __forceinline__ void write_nothing(const SampleArgs &a, long r) {  // (nothing to draw from)
    a.classes[r] = -1;
    if (a.log_prob) a.log_prob[r] = -INFINITY;
}

// Sums of value(logit, index) by pieces and over what the workgroup holds; wave[w]: LDS, the part of wave w.
template <int THREADS, typename T, int N, typename F>
__device__ u64 sum_values(const HeldRow<T, N> &row, u64 (&own)[N], u64 *wave, F value) {
    u64 sum = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        own[i] = 0;
        if (i < row.rounds) {
            const int j = row.index(i);
            float v[HeldRow<T, N>::PER];
            unpack<T>(row.raw[i], v);
#pragma unroll
            for (int e = 0; e < HeldRow<T, N>::PER; ++e) own[i] += value(v[e], j + e);
            apart();
        }
        sum += own[i];
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    return sum_across<THREADS / 64>(wave);
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

// ------------------------------------------------------------------ a row in the registers of a workgroup

// 1 x 1000 with all filters: 7 us, 16 x 1000 without: 5 (a launch that does nothing takes 2 to 3): the histogram, two scans and the sums
// wait for each other, a row being one workgroup's.  256 x 16000: 18 us, in parts 34.
template <typename T, int N, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void sample_held_kernel(SampleArgs a, int row0) {
    __shared__ SearchLds s;
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    HeldRow<T, N> row(a.in, r, wave, THREADS / 64, lane);
    const Draw draw(a, r);
    float best = largest<THREADS>(row, s.part_f);
    if (best == -INFINITY) {
        if (threadIdx.x == 0) write_nothing(a, r);
        return;
    }
    const double inv_t = 1.0 / (double)draw.temperature;
    const bool infinite = best == INFINITY;
    if (infinite) row.only_infinite(), best = 0.0f;
    Kept kept{Weight(best, inv_t), keep_all(), draw.t_min(), fraction_bits(a.in.n)};
    if (draw.cuts(a.in.n)) {
        constexpr int OWN = BINS / THREADS;
        const Grid grid(best, inv_t, best);  // (the largest logit is place 0: a row of equal logits has exact sums, and its cut is where the count says)
        const Packed packed(a.in.n);
        if (threadIdx.x == 0) s.before = 0, s.weight_before = 0;
        build_histogram<THREADS>(row, grid, packed, s);
        uint32_t count[OWN];
        u64 lacking[OWN];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const u64 v = s.weight[threadIdx.x * OWN + i];
            count[i] = packed.count(v), lacking[i] = packed.lack(v);
        }
        Limit limit{(uint32_t)draw.k, INFINITY};
        const Range f = search<THREADS>(s, grid, packed, best, limit, draw, kept.t_min, count, lacking, 0, kept.fraction);
        if (f.start < BINS) {
            Row<T> whole(a.in, r, wave, THREADS / 64, lane);
            if (infinite) whole.only_infinite();
            kept.cut = cut_among<THREADS, true>(row, whole, kept.weight, s, limit, f.low, f.high, kept.fraction);
        }
    }
    u64 own[N];
    const u64 total = sum_values<THREADS>(row, own, s.part64, kept);
    first_beyond<THREADS>(row, own, s.part64, target_of(draw.u, total), kept, [&](float z, int j) { write_answer(a, r, j, kept.weight.log2_of(z), kept.fraction, total); });
}

// ------------------------------------------------------------------ a row in parts

// 512 x 100003 in float32, top_p, min_p and temperature: 125 us, in launches of 53, 13, 37 and 25.  The first reads the row (206 MB, floor
// 41) and adds to a histogram in LDS, 17 instructions of 64 bits a logit; the third reads it again, at 6 TB/s, to list one interval's members:
// the row fits no compute unit's registers.  1 x 131071 in bf16: 5, 12, 5 and 9 us, of which the second and the last are one workgroup's.
constexpr int PART_THREADS = 256, JOIN_THREADS = 1024;
// Members of the interval in which a row is cut that are kept for its last step.  Where it has more (flat rows, high temperatures, hundreds of
// thousands of classes) the last launch's one workgroup reads the row itself for every step instead: normal logits, deviation 2.5, top_p
// 0.95, 16 x 250007: 42 us at T = 1, 254 at T = 2; 4 x 1048576: 753 and 940.
constexpr int LIST = 4096;
constexpr int MOST_PARTS = LOGITS_MOST_PARTS;

// What a part has of its row: its maximum and how often; the histogram over a grid that all parts of the row share (place 0 is the
// logit 0), from the maximum's interval on, without what equals the maximum; or, without filters, the sum of its weights.
struct SamplePart {
    float best;
    uint32_t equal, ordered;  // logits that equal the maximum, that are above -inf
    int used;                 // intervals up to the last that is not empty; what is behind is not written
    double top, sum;
    u64 kept;  // sum of the weights that are kept whatever the list says
    u64 weight[BINS];
};
// What the parts need to know of their row once the histograms are joined.
struct SampleRow {
    float best;
    int start;           // the interval in which the row is cut (Range)
    uint32_t low, high;
    uint32_t before, inside;
    u64 weight_before;
    double limit;
    int n;  // listed
    u64 entry[LIST];
};

template <typename T, int PIECES, int THREADS>
using PartRow = HeldRow<T, (PIECES + THREADS - 1) / THREADS>;
template <typename T, int PIECES, int THREADS>
__device__ __forceinline__ PartRow<T, PIECES, THREADS> part_row(const SampleArgs &a, long r, int part) {
    // (a workgroup with more threads than pieces: waves without any)
    constexpr int WAVES = PIECES < THREADS ? PIECES / 64 : THREADS / 64;
    const int wave = threadIdx.x >> 6;
    PartRow<T, PIECES, THREADS> row(a.in, r, wave < WAVES ? wave : 0, WAVES, threadIdx.x & 63, part * PIECES, PIECES);
    if (wave >= WAVES) row.rounds = 0;
    return row;
}

// First launch.  CUT: histograms; else sums.
template <typename T, int PIECES, bool CUT>
__global__ __launch_bounds__(PART_THREADS) void sample_part_kernel(SampleArgs a, int row0, int parts, SamplePart *out) {
    __shared__ SearchLds s;
    __shared__ double part_d[PART_THREADS / 64];
    const long r = (long)row0 + blockIdx.x / parts;
    PartRow<T, PIECES, PART_THREADS> row = part_row<T, PIECES, PART_THREADS>(a, r, blockIdx.x % parts);
    const Draw draw(a, r);
    SamplePart &mine = out[blockIdx.x];
    const float m = largest<PART_THREADS>(row, s.part_f);
    const float best = m == INFINITY ? 0.0f : m;
    if (threadIdx.x == 0) mine.best = m;
    if (m == -INFINITY) return;
    if (m == INFINITY) row.only_infinite();
    const double inv_t = 1.0 / (double)draw.temperature;
    if (!CUT) {
        const Weight weight(best, inv_t);
        double sum = 0.0;
        row.each([&](float z, int) { sum += exp2_64<11>(weight.log2_of(z)); });
        sum = block_sum<PART_THREADS>(sum, part_d);
        if (threadIdx.x == 0) mine.sum = sum;
        return;
    }
    const Grid grid(best, inv_t, 0.0);
    const Packed packed(LOGITS_PART_PIECES * (16 / (int)sizeof(T)));
    build_histogram<PART_THREADS>(row, grid, packed, s);
    uint32_t equal = 0;
    row.each([&](float z, int) { equal += __popcll(__ballot(z == best)); });  // (of the wave)
    uint32_t ordered = 0;
    int used = 0;
    for (int b = threadIdx.x; b < BINS; b += PART_THREADS) {
        const uint32_t n = packed.count(s.weight[b]);
        ordered += n, used = n ? b + 1 : used;
    }
    ordered = wave_sum(ordered), used = wave_all(used, [](int p, int q) { return p > q ? p : q; });
    if ((threadIdx.x & 63) == 0) s.part32[threadIdx.x >> 6] = equal, s.part32[4 + (threadIdx.x >> 6)] = ordered, s.count[threadIdx.x >> 6] = used;
    __syncthreads();
    equal = s.part32[0] + s.part32[1] + s.part32[2] + s.part32[3], ordered = s.part32[4] + s.part32[5] + s.part32[6] + s.part32[7];
    used = max(max(s.count[0], s.count[1]), max(s.count[2], s.count[3]));
    const double t = grid.place(best);
    for (int b = threadIdx.x; b < used; b += PART_THREADS) mine.weight[b] = s.weight[b] - (b == 0 ? equal * packed.one(t - floor(t)) : 0);
    if (threadIdx.x == 0) mine.equal = equal, mine.ordered = ordered, mine.used = used, mine.top = grid.top;
}

// Second launch, a workgroup per row: the joined histogram, and where the row is cut.
__global__ __launch_bounds__(JOIN_THREADS) void sample_join_kernel(SampleArgs a, int row0, int parts, const SamplePart *in, SampleRow *out) {
    __shared__ SearchLds s;
    __shared__ int down[MOST_PARTS], used[MOST_PARTS];
    __shared__ uint32_t sums[2];
    static_assert(BINS == JOIN_THREADS, "a thread has one interval");
    const long r = (long)row0 + blockIdx.x;
    in += (long)blockIdx.x * parts;
    SampleRow &row = out[blockIdx.x];
    const Draw draw(a, r);
    float part_best = -INFINITY;
    double top = 0.0;
    uint32_t part_equal = 0, part_ordered = 0;
    int part_used = 0;
    if ((int)threadIdx.x < parts) {
        const SamplePart &p = in[threadIdx.x];
        part_best = p.best, top = p.top, part_equal = p.equal, part_ordered = p.ordered, part_used = p.used;
    }
    s.count[threadIdx.x] = 0, s.weight[threadIdx.x] = 0;
    if (threadIdx.x < 2) sums[threadIdx.x] = 0;
    const float m = block_all<JOIN_THREADS>(part_best, s.part_f, [](float p, float q) { return fmaxf(p, q); });
    if (threadIdx.x == 0) row.best = m, row.n = 0, row.start = BINS, s.before = 0, s.weight_before = 0;
    if (m == -INFINITY || !draw.cuts(a.in.n)) return;
    const float best = m == INFINITY ? 0.0f : m;
    const int fraction = fraction_bits(a.in.n);
    const Grid grid(best, 1.0 / (double)draw.temperature, 0.0);
    const Packed packed(LOGITS_PART_PIECES * (a.in.bf16 ? 8 : 4));
    if ((int)threadIdx.x < parts) {
        const bool counts = part_best > -INFINITY && (m < INFINITY || part_best == INFINITY);
        // the part's intervals lie that much further down
        const int d = counts ? (int)fmin(top - grid.top, (double)BINS) : BINS;
        down[threadIdx.x] = d, used[threadIdx.x] = part_used;
        if (counts) {
            atomicAdd(&sums[0], part_ordered);
            if (part_best == m) {
                atomicAdd(&sums[1], part_equal);
            } else if (d < BINS - 1) {  // what equals the part's maximum, at its own place
                const double t = grid.place(part_best);
                atomicAdd(&s.count[d], part_equal);
                atomicAdd(&s.weight[d], part_equal * packed.lack(packed.one(t - floor(t))));
            }
        }
    }
    __syncthreads();
    uint32_t count[1] = {0};
    u64 lacking[1] = {0};
    constexpr int BATCH = 16;  // (their loads are on the way together)
    for (int first = 0; first < parts; first += BATCH) {
        u64 v[BATCH];
        const int p_lane = min(first + (int)(threadIdx.x & (BATCH - 1)), parts - 1), down_lane = down[p_lane], used_lane = used[p_lane];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int b = (int)threadIdx.x - read_lane(down_lane, i);
            v[i] = 0;
            if (first + i < parts && b >= 0 && b < read_lane(used_lane, i)) v[i] = in[first + i].weight[b];
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) count[0] += packed.count(v[i]), lacking[0] += packed.lack(v[i]);
    }
    const uint32_t ordered = sums[0], equal = sums[1];
    count[0] = threadIdx.x < BINS - 1 ? count[0] + s.count[threadIdx.x] : 0;
    lacking[0] += s.weight[threadIdx.x];
    // what falls off the end, in the last interval
    const uint32_t placed = block_sum<JOIN_THREADS>(count[0], s.part32);
    if (threadIdx.x == BINS - 1) count[0] = ordered - placed - equal;
    __syncthreads();
    Limit limit{(uint32_t)draw.k, INFINITY};
    const Range f = search<JOIN_THREADS>(s, grid, packed, best, limit, draw, draw.t_min(), count, lacking, equal, fraction);
    if (threadIdx.x == 0) {
        row.start = f.start, row.low = f.low, row.high = f.high;
        row.before = s.before, row.inside = s.inside, row.weight_before = s.weight_before, row.limit = limit.weight;
    }
}

// Third launch: each part lists its members of that interval, and sums the weights above it (from its histogram).
template <typename T, int PIECES>
__global__ __launch_bounds__(PART_THREADS) void sample_gather_kernel(SampleArgs a, int row0, int parts, SamplePart *part_out, SampleRow *rows) {
    __shared__ double part_d[PART_THREADS / 64];
    __shared__ int n, at;
    constexpr int OWN = BINS / PART_THREADS;
    const long r = (long)row0 + blockIdx.x / parts;
    SampleRow &state = rows[blockIdx.x / parts];
    SamplePart &mine = part_out[blockIdx.x];
    PartRow<T, PIECES, PART_THREADS> row = part_row<T, PIECES, PART_THREADS>(a, r, blockIdx.x % parts);
    const int used = mine.used;
    u64 v[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        v[i] = 0;
        if (i * PART_THREADS + (int)threadIdx.x < used) v[i] = mine.weight[i * PART_THREADS + threadIdx.x];
    }
    const float m = state.best, part_best = mine.best;
    const uint32_t low = state.low, high = state.high;
    const int start = state.start;
    const Draw draw(a, r);
    if (part_best == -INFINITY || (m == INFINITY && part_best < INFINITY)) {  // (nothing here)
        if (threadIdx.x == 0) mine.kept = 0;
        return;
    }
    if (m == INFINITY) row.only_infinite();
    const float best = m == INFINITY ? 0.0f : m, own_best = part_best == INFINITY ? 0.0f : part_best;
    const double inv_t = 1.0 / (double)draw.temperature;
    const Grid grid(best, inv_t, 0.0);
    const Packed packed(LOGITS_PART_PIECES * (16 / (int)sizeof(T)));
    const int fraction = fraction_bits(a.in.n);
    if (threadIdx.x == 0) n = 0;
    // weights of the part's intervals before the row's `start`
    const double down = mine.top - grid.top, above = grid.place(best) - grid.top;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int b = i * PART_THREADS + threadIdx.x;
        if (v[i] && b < BINS - 1 && b + down < start)
            sum += packed.sum(packed.count(v[i]), packed.lack(v[i])) * exp2_64<11>((above - down - b) * (1.0 / BINS_PER_LOG2));
    }
    if (threadIdx.x == 0 && down < start) sum += mine.equal * exp2_64<11>(Weight(best, inv_t).log2_of(own_best));
    sum = block_sum<PART_THREADS>(sum, part_d);
    if (threadIdx.x == 0) mine.kept = (u64)ldexp(sum, fraction);
    if (start >= BINS || !(own_best >= key_value(low))) return;
    int members = 0;
    row.each([&](float z, int) {
        const uint32_t k = order_key(z);
        members += k >= low && k <= high;
    });
    // a run of the row's list for them
    int before = wave_scan(members);
    const int all = __shfl(before, 63), lane = threadIdx.x & 63;
    int wave_at = 0;
    if (lane == 0 && all) wave_at = atomicAdd(&n, all);
    before += __shfl(wave_at, 0) - members;
    __syncthreads();
    if (threadIdx.x == 0 && n) at = atomicAdd(&state.n, n);
    __syncthreads();
    before += at;
    if (members)
        row.each_from(key_value(low), [&](float z, int j) {
            const uint32_t k = order_key(z);
            if (k <= high) {
                if (before < LIST) state.entry[before] = (u64)k << 32 | (uint32_t)j;
                ++before;
            }
        });
}

// A row's list, in registers.
struct Listed {
    static constexpr int OWN = LIST / JOIN_THREADS;
    u64 entry[OWN];
    __device__ __forceinline__ void load(const u64 *from) {  // (whether or not there is something: the loads need not wait for the number)
#pragma unroll
        for (int i = 0; i < OWN; ++i) entry[i] = from[i * JOIN_THREADS + threadIdx.x];
    }
    __device__ __forceinline__ void limit_to(int n) {
#pragma unroll
        for (int i = 0; i < OWN; ++i) entry[i] = i * JOIN_THREADS + (int)threadIdx.x < n ? entry[i] : 0;
    }
    template <typename F>
    __device__ __forceinline__ void each_from(float z_low, F f) const {
        const uint32_t low = order_key(z_low);
#pragma unroll
        for (int i = 0; i < OWN; ++i)
            if ((uint32_t)(entry[i] >> 32) >= low) f(key_value((uint32_t)(entry[i] >> 32)), (int)(uint32_t)entry[i]);
    }
};

// Last launch, a workgroup per row: the cut, the part in which the running sum passes the target, and the class there.  With 89
// registers a compute unit has room for one workgroup (CUT): 512 rows take two rounds.
template <typename T, int PIECES, bool CUT>
__global__ __launch_bounds__(JOIN_THREADS) void sample_finish_kernel(SampleArgs a, int row0, int parts, const SamplePart *in, const SampleRow *rows) {
    __shared__ SearchLds s;
    __shared__ u64 sums[MOST_PARTS];
    __shared__ int chosen;
    __shared__ u64 chosen_before, all_parts;
    constexpr int PER = 16 / sizeof(T);
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    in += (long)blockIdx.x * parts;
    Listed listed;
    if (CUT) listed.load(rows[blockIdx.x].entry);
    const Draw draw(a, r);
    Row<T> whole(a.in, r, wave, JOIN_THREADS / 64, lane);
    float m = -INFINITY;
    u64 part_kept = 0;
    if ((int)threadIdx.x < parts) {
        m = in[threadIdx.x].best;
        if (CUT) part_kept = in[threadIdx.x].kept;
    }
    const float mine = m;
    m = block_all<JOIN_THREADS>(m, s.part_f, [](float p, float q) { return fmaxf(p, q); });
    if (m == -INFINITY) {
        if (threadIdx.x == 0) write_nothing(a, r);
        return;
    }
    if (m == INFINITY) whole.only_infinite();
    const float best = m == INFINITY ? 0.0f : m;
    Kept kept{Weight(best, 1.0 / (double)draw.temperature), keep_all(), draw.t_min(), fraction_bits(a.in.n)};
    if (CUT) {
        const SampleRow &state = rows[blockIdx.x];
        const uint32_t low = state.low, high = state.high;
        const int start = state.start;
        if (threadIdx.x == 0) s.before = state.before, s.weight_before = state.weight_before, s.inside = state.inside;
        if ((int)threadIdx.x < parts) sums[threadIdx.x] = part_kept;
        __syncthreads();
        if (start < BINS) {
            const Limit limit{(uint32_t)draw.k, state.limit};
            const bool all = state.n <= LIST;
            listed.limit_to(state.n);
            kept.cut = all ? cut_among<JOIN_THREADS, true>(listed, whole, kept.weight, s, limit, low, high, kept.fraction)
                                        : cut_among<JOIN_THREADS, true>(whole, whole, kept.weight, s, limit, low, high, kept.fraction);
            // the kept members, to the sums of their parts
            auto add = [&](float z, int j) {
                const uint32_t k = order_key(z);
                if (k >= low && k <= high) atomicAdd(&sums[(j + whole.lead) / (PIECES * PER)], kept(z, j));
            };
            if (all)
                listed.each_from(key_value(low), add);
            else
                whole.each_from(key_value(low), add);
        }
    } else {
        if ((int)threadIdx.x < parts) {
            const float z = m == INFINITY ? as_infinite(mine) : mine;
            const double t = kept.weight.log2_of(z);
            sums[threadIdx.x] = z > -INFINITY ? (u64)ldexp(in[threadIdx.x].sum * exp2_64<11>(t), kept.fraction) : 0;
        }
        if (draw.first) {  // (no histogram was asked for: the first of the largest)
            int j = 0x7FFFFFFF;
            whole.each([&](float z, int at) { j = min(j, z == best ? at : 0x7FFFFFFF); });
            __syncthreads();
            j = block_all<JOIN_THREADS>(j, reinterpret_cast<int *>(s.part32), [](int p, int q) { return p < q ? p : q; });
            if (threadIdx.x == 0) {
                a.classes[r] = j;
                if (a.log_prob) a.log_prob[r] = 0.0f;
            }
            return;
        }
    }
    __syncthreads();
    if (wave == 0) {  // the part
        u64 total = 0;
        for (int p = lane; p < parts; p += 64) total += sums[p];
        total = wave_sum(total);
        const u64 target = target_of(draw.u, total);
        u64 before = 0;
        for (int p = 0; p < parts; p += 64) {
            const u64 own = p + lane < parts ? sums[p + lane] : 0, upto = before + wave_scan(own);
            if (upto > target && upto - own <= target) chosen = p + lane, chosen_before = upto - own;
            before = __shfl(upto, 63);
        }
        if (lane == 0) all_parts = total;
    }
    __syncthreads();
    const u64 total = all_parts, target = target_of(draw.u, total), before = chosen_before;
    PartRow<T, PIECES, JOIN_THREADS> row = part_row<T, PIECES, JOIN_THREADS>(a, r, chosen);
    if (m == INFINITY) row.only_infinite();
    u64 own[(PIECES + JOIN_THREADS - 1) / JOIN_THREADS];
    const u64 here = sum_values<JOIN_THREADS>(row, own, s.part64, kept);
    if (here == 0) {  // (a part whose weights are all below the point by themselves, if not by their sum: its largest)
        const float part_best = m == INFINITY ? 0.0f : in[chosen].best;
        int j = 0x7FFFFFFF;
        row.each([&](float z, int at) { j = min(j, z == part_best ? at : 0x7FFFFFFF); });
        j = block_all<JOIN_THREADS>(j, reinterpret_cast<int *>(s.part32), [](int p, int q) { return p < q ? p : q; });
        if (threadIdx.x == 0) write_answer(a, r, j, kept.weight.log2_of(part_best), kept.fraction, total);
        return;
    }
    // (sums made in another way may differ by a rounding: the last of the part then)
    first_beyond<JOIN_THREADS>(row, own, s.part64, min(target - before, here - 1), kept,
                               [&](float z, int j) { write_answer(a, r, j, kept.weight.log2_of(z), kept.fraction, total); });
}

bool cuts(const SampleArgs &a) { return a.top_k || a.top_p || a.min_p; }

// most: rows of a launch.
template <typename T, int PIECES>
hipError_t launch_parts(const SampleArgs &a, int pieces, long most, char *ws, hipStream_t s) {
    const int parts = logits_parts(pieces, PIECES);
    SampleRow *rows = reinterpret_cast<SampleRow *>(ws);
    SamplePart *sums = reinterpret_cast<SamplePart *>(ws + most * sizeof(SampleRow));
    return by_slices(a.in.rows, most, [&](int r, int n) {
        if (cuts(a)) {
            sample_part_kernel<T, PIECES, true><<<n * parts, PART_THREADS, 0, s>>>(a, r, parts, sums);
            sample_join_kernel<<<n, JOIN_THREADS, 0, s>>>(a, r, parts, sums, rows);
            sample_gather_kernel<T, PIECES><<<n * parts, PART_THREADS, 0, s>>>(a, r, parts, sums, rows);
            sample_finish_kernel<T, PIECES, true><<<n, JOIN_THREADS, 0, s>>>(a, r, parts, sums, rows);
        } else {
            sample_part_kernel<T, PIECES, false><<<n * parts, PART_THREADS, 0, s>>>(a, r, parts, sums);
            sample_finish_kernel<T, PIECES, false><<<n, JOIN_THREADS, 0, s>>>(a, r, parts, sums, rows);
        }
    });
}

template <typename T>
hipError_t launch(const SampleArgs &a, char *ws, hipStream_t s) {
    const int pieces = logits_pieces(a.in.n, a.in.bf16);
    if (cuts(a) ? held_rows(a.in) : held_plain_rows(a.in))
        return by_size(pieces, [&](auto N, auto THREADS) {
            return by_slices(a.in.rows, (1l << 31) / THREADS, [&](int r, int n) { sample_held_kernel<T, decltype(N)::value, decltype(THREADS)::value><<<n, (int)THREADS, 0, s>>>(a, r); });
        });
    if (small_parts(a.in, cuts(a) ? LOGITS_FEW_PARTS : LOGITS_MOST_PARTS)) return launch_parts<T, LOGITS_SMALL_PART_PIECES>(a, pieces, a.in.rows, ws, s);
    return launch_parts<T, LOGITS_PART_PIECES>(a, pieces, rows_of_slice(a.in.n) < a.in.rows ? rows_of_slice(a.in.n) : a.in.rows, ws, s);
}

}  // namespace

size_t sample_part_bytes() { return sizeof(SamplePart); }
size_t sample_row_bytes() { return sizeof(SampleRow); }

hipError_t launch_sample(const SampleArgs &a, void *ws, hipStream_t s) { return a.in.bf16 ? launch<uint16_t>(a, static_cast<char *>(ws), s) : launch<float>(a, static_cast<char *>(ws), s); }

}  // namespace sushi
