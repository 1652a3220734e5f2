// The leading logits of a row and the probability mass outside them (logits.h).
//
// The row's groups (what a thread holds, or a 16-byte piece) have maxima; the k-th largest of these maxima is reached by k logits at
// least, so what lies below it is not among the first k.  Little reaches it: 70 logits of 32001 with k = 64 and 512 groups.  Those are
// listed in LDS, ranked, and the first k of them are the answer.  The mass outside is summed by itself, in 64 bits.
// A list that is too long (many equal logits) is cut by histograms of the keys (row_order.h).
#include "row_order.h"

namespace sushi {

namespace {

constexpr int TOP_LIST = 2 * LOGITS_MAX_TOP;

// A key that at least k of the keys reach (KEY_NONE + 1 if fewer are above that of -inf), close to the largest such.  For a whole wave, on
// keys in LDS, EACH a lane.
template <int EACH>
__device__ __forceinline__ uint32_t reached_by(const uint32_t *keys, int k) {
    uint32_t own[EACH], low = 0xFFFFFFFFu, high = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        own[e] = keys[e * 64 + (threadIdx.x & 63)];
        low = min(low, own[e]), high = max(high, own[e]);
    }
    auto count = [&](uint32_t key) {
        int n = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) n += __popcll(__ballot(own[e] >= key));
        return n;
    };
    low = max(wave_all(low, [](uint32_t a, uint32_t b) { return a < b ? a : b; }), KEY_NONE + 1);
    high = wave_all(high, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
    if (count(low) < k) return KEY_NONE + 1;
    for (int i = 0; i < 20 && low < high; ++i) {
        const uint32_t middle = low + (high - low) / 2 + 1;
        const int n = count(middle);
        if (n >= k) low = middle; else high = middle - 1;
        if (n == k) break;
    }
    return low;
}

struct Order {
    union {
        u64 entry[TOP_LIST];  // keys above inverted indexes
        uint32_t maxima[LOGITS_PART_PIECES];
        SearchLds s;
    };
    int n;
    uint32_t bound;
};
__device__ __forceinline__ u64 entry_of(uint32_t key, int j) { return (u64)key << 32 | (uint32_t)~j; }
__device__ __forceinline__ uint32_t entry_key(u64 v) { return (uint32_t)(v >> 32); }

// put(place, entry) for every logit of the row that is at least z_low, which becomes -inf there; places in the order of threads and their
// pieces (not of an atomic: sums over the list are the same in every run).  Only the first TOP_LIST are put.  Returns how many there
// are.  part: LDS, an entry per wave.
template <int THREADS, typename T, int N, typename F>
__device__ __forceinline__ int take_out(HeldRow<T, N> &row, float z_low, int *part, F put) {
    constexpr int PER = HeldRow<T, N>::PER;
    static_assert(N * PER <= 64, "a mark for each logit of a thread");
    u64 marks = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < row.rounds) {
            float v[PER];
            unpack<T>(row.raw[i], v);
            bool any = false;
#pragma unroll
            for (int e = 0; e < PER; ++e) any |= v[e] >= z_low;
            if (any) {
                uint32_t some = 0;
#pragma unroll
                for (int e = 0; e < PER; ++e) some |= v[e] >= z_low ? 1u << e : 0u;
                marks |= (u64)some << (i * PER);
            }
        }
    const int own = __popcll(marks), upto = wave_scan(own);
    if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = upto;
    __syncthreads();
    int at = sum_before<THREADS / 64>(part) + upto - own;
    if (own > 0)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t some = (uint32_t)(marks >> (i * PER)) & ((1u << PER) - 1);
            if (some) {
                const uint4 r = row.raw[i];
                float v[PER];
                unpack<T>(r, v);
#pragma unroll
                for (int e = 0; e < PER; ++e) v[e] = some >> e & 1 ? -INFINITY : v[e];
                row.raw[i] = pack<T>(v);
                for (; some; some &= some - 1, ++at) {
                    const int e = __ffs(some) - 1;
                    if (at < TOP_LIST) put(at, entry_of(order_key(element<T>(r, e)), row.index(i) + e));
                }
            }
        }
    return sum_across<THREADS / 64>(part);
}

// Sorts SIZE entries, largest first: a bitonic network.  The 64 pairs of a wave lie in 128 neighbouring entries while the distance is at
// most 64: those steps need no barrier of the workgroup (64 x 2000, k = 1024: 36 us with one for each step and a pair at a time, 29.5 so).
template <int THREADS, int SIZE>
__device__ __forceinline__ void sort_entries(Order &o) {
    constexpr int OWN = (SIZE / 2 + THREADS - 1) / THREADS;
    for (int width = 2; width <= SIZE; width *= 2)
        for (int d = width / 2; d > 0; d /= 2) {
            u64 p[OWN], q[OWN];
            int lo[OWN];
#pragma unroll
            for (int t = 0; t < OWN; ++t) {
                const int i = min(t * THREADS + (int)threadIdx.x, SIZE / 2 - 1);
                lo[t] = (i & ~(d - 1)) * 2 + (i & (d - 1));
                p[t] = o.entry[lo[t]], q[t] = o.entry[lo[t] + d];
            }
#pragma unroll
            for (int t = 0; t < OWN; ++t)
                if (t * THREADS + (int)threadIdx.x < SIZE / 2) {
                    const bool turn = (p[t] < q[t]) == ((lo[t] & width) == 0);
                    o.entry[lo[t]] = turn ? q[t] : p[t], o.entry[lo[t] + d] = turn ? p[t] : q[t];
                }
            if (d > 64 || (d == 1 && width > 64))  // (the next step's distance: d / 2, or width)
                __syncthreads();
            else
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"), __builtin_amdgcn_wave_barrier();
        }
}

// Ranks the list (n entries) and writes the first k as the row's answer; adds the others' weights to outside, theirs to inside.
template <int THREADS>
__device__ __forceinline__ void write_first(const TopArgs &a, long r, Order &o, int n, const Weight &weight, bool infinite, double &inside, double &outside) {
    auto put = [&](int rank, u64 v) {
        const float z = key_value(entry_key(v));
        const double w = exp2_64<6>(weight.log2_of(infinite ? as_infinite(z) : z));
        const bool in = rank < a.k;  // (a branch between two sums would put both into memory)
        inside += in ? w : 0.0, outside += in ? 0.0 : w;
        if (in) a.values[r * a.k + rank] = z, a.classes[r * a.k + rank] = (int)~(uint32_t)v;
    };
    if (n <= 256) {  // (64 x 1000, k = 64: 8.2 us, sorted 13.8; with more entries the sort is level or ahead)
        // counted by as many neighbouring lanes for an entry as there are threads for
        static_assert(THREADS >= 256, "a lane for an entry at least");
        const int by = n * 16 <= THREADS ? 16 : n * 4 <= THREADS ? 4 : 1, lane = threadIdx.x & (by - 1), i = threadIdx.x / by;
        const u64 v = o.entry[min(i, TOP_LIST - 1)];
        int rank = 0;
        if (i < n) {
#pragma unroll 4
            for (int e = lane; e < n; e += by) rank += o.entry[e] > v;
            for (int d = 1; d < by; d *= 2) rank += __shfl_xor(rank, d);
        }
        __syncthreads();
        if (i < n && lane == 0) o.entry[rank] = v;
        __syncthreads();
    } else {
        const int size = n <= 512 ? 512 : n <= 1024 ? 1024 : TOP_LIST;
        for (int i = n + threadIdx.x; i < size; i += THREADS) o.entry[i] = 0;
        __syncthreads();
        if (size == 512)
            sort_entries<THREADS, 512>(o);
        else if (size == 1024)
            sort_entries<THREADS, 1024>(o);
        else
            sort_entries<THREADS, TOP_LIST>(o);
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += THREADS) put(i, o.entry[i]);  // (by rank: the sums are the same in every run)
    for (int i = n + threadIdx.x; i < a.k; i += THREADS) a.values[r * a.k + i] = -INFINITY, a.classes[r * a.k + i] = -1;
}

// The list from a source with more than TOP_LIST logits that reach the bound: exactly the first k; the rest's weights as they are
// below the cut, from the whole row.  n: how many reach the bound.
template <int THREADS, typename T>
__device__ __forceinline__ void list_exactly(const TopArgs &a, const Row<T> &row, Order &o, uint32_t low, int n, const Weight &weight, bool infinite, double *outside) {
    __syncthreads();
    if (threadIdx.x == 0) o.s.before = 0, o.s.weight_before = 0, o.s.inside = n, o.n = 0;
    __syncthreads();
    const Cut cut = cut_among<THREADS, false>(row, row, weight, o.s, Limit{(uint32_t)a.k, INFINITY}, low, 0xFF800000u, 0);
    __syncthreads();  // (the entries lie where the search was)
    double sum = 0.0;
    row.each([&](float z, int j) {
        const uint32_t k = order_key(z);
        if (k != KEY_NONE && cut.keeps(k, j))
            o.entry[min(atomicAdd(&o.n, 1), TOP_LIST - 1)] = entry_of(k, j);
        else
            sum += exp2_64<6>(weight.log2_of(infinite ? as_infinite(z) : z));
    });
    *outside = sum;
    __syncthreads();
}

// 2048 x 32001 in bf16, k = 64: 73 us, 131 MB, floor 26.  33 of it read the row and find the bound, 11 list and rank, 29 are the weights
// of the rest: 16 instructions of 64 bits a logit, which is what bounds it (without `rest`: 44).  Rows follow each other in few
// workgroups, the next one's loads ahead of this one's weights: 109 (128 registers); 1024 threads with half the pieces: 90.
template <typename T, int N, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS < 1024 ? 8 : 4) void top_held_kernel(TopArgs a, int row0) {
    __shared__ Order o;
    __shared__ double part[2][16];
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    HeldRow<T, N> row(a.in, r, wave, THREADS / 64, lane);
    float m = -INFINITY;
    row.each([&](float z, int) { m = fmaxf(m, z); });
    o.maxima[threadIdx.x] = order_key(m);
    __syncthreads();
    if (wave == 0) {
        const uint32_t bound = reached_by<THREADS / 64>(o.maxima, a.k);
        if (lane == 0) o.bound = bound;
    }
    uint32_t best = 0;
#pragma unroll
    for (int e = 0; e < THREADS / 64; ++e) best = max(best, o.maxima[e * 64 + lane]);
    best = wave_all(best, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    __syncthreads();
    const uint32_t bound = o.bound;
    const bool infinite = key_value(best) == INFINITY;
    const Weight weight(infinite ? 0.0f : key_value(best), 1.0 / (double)a.temperature);
    // what reaches the bound is listed and taken out of the row
    __shared__ int part_n[THREADS / 64];
    int n = take_out<THREADS>(row, key_value(bound), part_n, [&](int at, u64 v) { o.entry[at] = v; });
    __syncthreads();
    double inside = 0.0, outside = 0.0;
    if (n > TOP_LIST) {
        const Row<T> whole(a.in, r, wave, THREADS / 64, lane);
        list_exactly<THREADS>(a, whole, o, bound, n, weight, infinite, &outside);
        n = o.n;
    } else if (a.rest) {
        if (infinite) row.only_infinite();
        row.each([&](float z, int) { outside += exp2_64<6>(weight.log2_of(z)); });
    }
    write_first<THREADS>(a, r, o, n, weight, infinite, inside, outside);
    if (!a.rest) return;
    inside = wave_sum(inside), outside = wave_sum(outside);
    if (lane == 0) part[0][wave] = inside, part[1][wave] = outside;
    __syncthreads();
    inside = sum_across<THREADS / 64>(part[0]), outside = sum_across<THREADS / 64>(part[1]);
    if (threadIdx.x == 0) a.rest[r] = inside > 0.0 ? (float)(outside / (inside + outside)) : 0.0f;
}

// ------------------------------------------------------------------ a row in parts

constexpr int PART_THREADS = 256, PART_ROUNDS = LOGITS_PART_PIECES / PART_THREADS, JOIN_THREADS = 1024;

// 3 x 200003 in float32, k = 100 (25 parts a row): 11 us, then 12 for the join of three workgroups, whose loads, list and ranks wait for
// each other.  512 x 131071 in bf16, k = 16: 105 us, without `rest` 67 (floor 26).  80 registers, so that six workgroups share a compute
// unit: with 143 for bf16, which is what the compiler takes by itself, 115 us.

// What a part has of the first k: what reaches the k-th largest of its own pieces' maxima.
struct TopPart {
    double outside;  // weights of the rest, at the part's own maximum
    uint32_t best;   // key of the maximum
    uint32_t bound;  // k logits of the part reach it, if it has as many
    uint32_t bound_some;  // share_of() logits of it do
    int n;           // listed; more than TOP_LIST: the list is not complete
    u64 entry[TOP_LIST];
};

// A part's share of the first k, twice: half of the parts have k logits above a bound that each reaches with so many.
__device__ __forceinline__ int share_of(int k, int parts) { return (2 * k + parts - 1) / parts; }

template <typename T>
__global__ __launch_bounds__(PART_THREADS, 6) void top_part_kernel(TopArgs a, int row0, int parts, TopPart *out) {
    __shared__ Order o;
    __shared__ double part_d[PART_THREADS / 64];
    const long r = (long)row0 + blockIdx.x / parts;
    const int part = blockIdx.x % parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    HeldRow<T, PART_ROUNDS> row(a.in, r, wave, PART_THREADS / 64, lane, part * LOGITS_PART_PIECES, LOGITS_PART_PIECES);
    constexpr int PER = HeldRow<T, PART_ROUNDS>::PER;
    // groups of 8, 4, 2 pieces or 1 of a thread: three times as many as k, if there are (the bound is loose with fewer, and finding
    // it takes longer with more)
    const int each = 3 * a.k <= PART_THREADS ? 8 : 3 * a.k <= 2 * PART_THREADS ? 4 : 3 * a.k <= 4 * PART_THREADS ? 2 : 1;
    uint32_t best = KEY_NONE, group = KEY_NONE;
#pragma unroll
    for (int i = 0; i < PART_ROUNDS; ++i) {
        float v[PER], m = -INFINITY;
        unpack<T>(row.raw[i], v);
#pragma unroll
        for (int e = 0; e < PER; ++e) m = fmaxf(m, v[e]);
        if (i < row.rounds) group = max(group, order_key(m));
        if ((i + 1) % each == 0) {
            o.maxima[i / each * PART_THREADS + threadIdx.x] = group;
            best = max(best, group), group = KEY_NONE;
        }
    }
    __syncthreads();
    __shared__ uint32_t bound_some;
    if (wave < 2) {  // (side by side)
        const int k = wave == 0 ? a.k : share_of(a.k, parts);
        const uint32_t bound = each == 8   ? reached_by<PART_THREADS / 64>(o.maxima, k)
                               : each == 4 ? reached_by<2 * PART_THREADS / 64>(o.maxima, k)
                               : each == 2 ? reached_by<4 * PART_THREADS / 64>(o.maxima, k)
                                           : reached_by<8 * PART_THREADS / 64>(o.maxima, k);
        if (lane == 0) (wave == 0 ? o.bound : bound_some) = bound;
    }
    best = wave_all(best, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    __shared__ uint32_t part_k[PART_THREADS / 64];
    if (lane == 0) part_k[wave] = best;
    __syncthreads();
    best = across_waves<PART_THREADS / 64>(part_k, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    TopPart &mine = out[blockIdx.x];
    __shared__ int part_n[PART_THREADS / 64];
    const int n = take_out<PART_THREADS>(row, key_value(o.bound), part_n, [&](int at, u64 v) { mine.entry[at] = v; });
    const bool infinite = key_value(best) == INFINITY;
    const Weight weight(infinite ? 0.0f : key_value(best), 1.0 / (double)a.temperature);
    double outside = 0.0;
    if (a.rest) {
        if (infinite) row.only_infinite();
        row.each([&](float z, int) { outside += exp2_64<6>(weight.log2_of(z)); });
    }
    outside = block_sum<PART_THREADS>(outside, part_d);
    if (threadIdx.x == 0) mine.outside = outside, mine.best = best, mine.bound = o.bound, mine.bound_some = bound_some, mine.n = n;
}

template <typename T>
__global__ __launch_bounds__(JOIN_THREADS) void top_join_kernel(TopArgs a, int row0, int parts, const TopPart *in) {
    __shared__ Order o;
    __shared__ int listed[LOGITS_MOST_PARTS];
    constexpr int EACH = (LOGITS_MOST_PARTS + 63) / 64;
    __shared__ uint32_t some[EACH * 64];
    __shared__ uint32_t part_k[2][JOIN_THREADS / 64];
    __shared__ int part_n[JOIN_THREADS / 64];
    __shared__ double part_d[2][JOIN_THREADS / 64];
    const long r = (long)row0 + blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    in += (long)blockIdx.x * parts;
    uint32_t best = 0, bound = 0, own_best = 0;
    int most = 0;
    double own_outside = 0.0;
    if ((int)threadIdx.x < parts) {
        const TopPart &p = in[threadIdx.x];
        own_best = best = p.best, bound = p.bound, own_outside = p.outside, most = p.n;
        listed[threadIdx.x] = min(most, TOP_LIST);
    }
    if (threadIdx.x < EACH * 64) some[threadIdx.x] = (int)threadIdx.x < parts ? in[threadIdx.x].bound_some : KEY_NONE;
    if (threadIdx.x == 0) o.n = 0;
    auto larger = [](uint32_t p, uint32_t q) { return p > q ? p : q; };
    best = wave_all(best, larger), bound = wave_all(bound, larger), most = wave_all(most, [](int p, int q) { return p > q ? p : q; });
    if (lane == 0) part_k[0][wave] = best, part_k[1][wave] = bound, part_n[wave] = most;
    __syncthreads();
    best = across_waves<JOIN_THREADS / 64>(part_k[0], larger);
    bound = across_waves<JOIN_THREADS / 64>(part_k[1], larger);  // (k logits of one part reach it)
    const int share = share_of(a.k, parts);
    bound = max(bound, reached_by<EACH>(some, (a.k + share - 1) / share));  // (that many parts, with so many each)
    most = across_waves<JOIN_THREADS / 64>(part_n, [](int p, int q) { return p > q ? p : q; });
    const bool infinite = key_value(best) == INFINITY;
    const Weight weight(infinite ? 0.0f : key_value(best), 1.0 / (double)a.temperature);
    auto weigh = [&](uint32_t key) { return exp2_64<11>(weight.log2_of(infinite ? as_infinite(key_value(key)) : key_value(key))); };
    double inside = 0.0, outside = own_outside > 0.0 ? own_outside * weigh(own_best) : 0.0;
    // what the parts have listed and reaches the bound
    if (most <= TOP_LIST) {
        int shift = 6;  // each part's list in so many places, four of them loaded at once
        while (1 << shift < most) ++shift;
        for (int i0 = threadIdx.x; i0 < parts << shift; i0 += 4 * JOIN_THREADS) {
            u64 v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + e * JOIN_THREADS, p = min(i >> shift, parts - 1), at = i & ((1 << shift) - 1);
                const bool there = i >> shift < parts && at < listed[p];
                v[e] = in[p].entry[there ? at : 0];
                v[e] = there ? v[e] : 0;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (entry_key(v[e]) >= bound) {
                    const int at = atomicAdd(&o.n, 1);
                    if (at < TOP_LIST) o.entry[at] = v[e];
                } else if (v[e]) {
                    outside += weigh(entry_key(v[e]));
                }
        }
    }
    __syncthreads();
    const int n = o.n;
    if (most > TOP_LIST || n > TOP_LIST) {  // (many equal logits)
        const Row<T> whole(a.in, r, wave, JOIN_THREADS / 64, lane);
        uint32_t reaching = 0;
        whole.each([&](float z, int) { reaching += z > -INFINITY && order_key(z) >= bound; });
        reaching = block_sum<JOIN_THREADS>(reaching, part_k[0]);
        list_exactly<JOIN_THREADS>(a, whole, o, bound, (int)reaching, weight, infinite, &outside);
    }
    write_first<JOIN_THREADS>(a, r, o, o.n, weight, infinite, inside, outside);
    if (!a.rest) return;
    inside = wave_sum(inside), outside = wave_sum(outside);
    if (lane == 0) part_d[0][wave] = inside, part_d[1][wave] = outside;
    __syncthreads();
    inside = sum_across<JOIN_THREADS / 64>(part_d[0]), outside = sum_across<JOIN_THREADS / 64>(part_d[1]);
    if (threadIdx.x == 0) a.rest[r] = inside > 0.0 ? (float)(outside / (inside + outside)) : 0.0f;
}

template <typename T>
hipError_t launch(const TopArgs &a, TopPart *ws, hipStream_t s) {
    if (held_rows(a.in))
        return by_size(logits_pieces(a.in.n, a.in.bf16), [&](auto N, auto THREADS) {
            return by_slices(a.in.rows, (1l << 31) / THREADS, [&](int r, int n) { top_held_kernel<T, decltype(N)::value, decltype(THREADS)::value><<<n, (int)THREADS, 0, s>>>(a, r); });
        });
    const int parts = logits_parts(logits_pieces(a.in.n, a.in.bf16), LOGITS_PART_PIECES);
    return by_slices(a.in.rows, rows_of_slice(a.in.n), [&](int r, int n) {
        top_part_kernel<T><<<n * parts, PART_THREADS, 0, s>>>(a, r, parts, ws);
        top_join_kernel<T><<<n, JOIN_THREADS, 0, s>>>(a, r, parts, ws);
    });
}

}  // namespace

size_t top_logits_part_bytes() { return sizeof(TopPart); }

hipError_t launch_top_logits(const TopArgs &a, void *ws, hipStream_t s) {
    return a.in.bf16 ? launch<uint16_t>(a, static_cast<TopPart *>(ws), s) : launch<float>(a, static_cast<TopPart *>(ws), s);
}

}  // namespace sushi
