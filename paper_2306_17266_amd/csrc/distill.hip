// Distillation from a teacher's leading logits (logits.h): the loss of a row and its gradient.
//
//   q = softmax(z / T);  e_j = exp((z_j - max z) / T), S = their sum, R = their sum over the classes that are not listed
//   p_i = (1 - r) softmax(t / T) over the row's list, r = the mass outside it
//   loss  = sum_i p_i (ln p_i - ln q_i) + r (ln r - ln(R / S))
//   d loss / d z_j = (e_j / S - p_j) / T for a listed class, e_j (1 / S - r / R) / T for another
//
// The loss is a small difference of large terms where student and teacher agree, and R is a small part of S where both are sure:
// R is summed by itself, never as S minus the list, and the sums, the list's terms and the logarithms have 64 bits.
#include <algorithm>

#include "logits_device.h"

namespace sushi {

namespace {

constexpr int THREADS = 256;
constexpr int PART_PIECES = LOGITS_PART_PIECES;
constexpr int LIST_BITS = 1 << 18;

// What a part of a row adds to it, and what a row's loss and gradient need, in the workspace.
struct PartSums {
    double rest;  // sum of the weights of what is not listed, at the part's own maximum
    float best;   // NaN if the part holds one
    float pad;
};
struct RowSums {
    double inv_sum;     // 1 / S
    double list_scale;  // (1 - r) / sum of exp((t - max t) / T)
    double rest_scale;  // weight (1 / S - r / R) / T
    float best, list_best;
    float weight;  // divided by T; 0: the gradient is zero
    float pad;
};

// Marks the row's listed classes in [low, high) (bit (class - low) & mask), and returns with *twice set if one may stand there twice.
// Entries outside are none of this workgroup's business.
__device__ void mark_list(const DistillArgs &a, long r, int low, int high, uint32_t mask, uint32_t *bits, int *list, int *twice) {
    for (uint32_t w = threadIdx.x; w <= mask >> 5; w += THREADS) bits[w] = 0;
    if (threadIdx.x == 0) *twice = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.k; i += THREADS) {
        const int c = a.classes[r * a.k + i];
        list[i] = c;
        if (c >= low && c < high) {
            const uint32_t b = (uint32_t)(c - low) & mask;
            if (atomicOr(&bits[b >> 5], 1u << (b & 31)) >> (b & 31) & 1) *twice = 1;
        }
    }
    __syncthreads();
}

// Whether entry i counts: its class exists, is in [low, high) and stands in no earlier entry.
__device__ __forceinline__ bool entry_counts(const int *list, int i, int low, int high, int twice) {
    const int c = list[i];
    if (c < low || c >= high) return false;
    for (int o = 0; twice && o < i; ++o)
        if (list[o] == c) return false;
    return true;
}

__device__ __forceinline__ int first_index(int part, int per, int lead) { return part * PART_PIECES * per - lead; }

template <typename T>
__device__ __forceinline__ float logit(const DistillArgs &a, long r, int c) {
    return ld1(static_cast<const T *>(a.in.x) + r * a.in.stride + c);
}

template <typename T>
__global__ __launch_bounds__(THREADS) void distill_part_kernel(DistillArgs a, int row0, int parts, PartSums *out) {
    constexpr int PER = 16 / sizeof(T), SPAN = PART_PIECES * PER;
    __shared__ uint32_t bits[SPAN / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    __shared__ float part_f[THREADS / 64];
    __shared__ double part_d[THREADS / 64];
    const long r = (long)row0 + blockIdx.x / parts;
    const int part = blockIdx.x % parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Row<T> row(a.in, r, wave, THREADS / 64, lane, part * PART_PIECES, PART_PIECES);
    const int low = first_index(part, PER, row.lead);
    mark_list(a, r, max(low, 0), min(low + SPAN, a.in.n), SPAN - 1, bits, list, &twice);
    const int base = max(low, 0);
    float m = -INFINITY;
    bool nan = false;
    row.each([&](float z, int) { m = fmaxf(m, z), nan |= z != z; });
    m = nan ? NAN : m;
    m = block_all<THREADS>(m, part_f, [](float x, float y) { return x != x || y != y ? NAN : fmaxf(x, y); });
    const Weight weight(m, 1.0 / (double)a.temperature);
    double rest = 0.0;
    row.each([&](float z, int j) {
        const uint32_t b = (uint32_t)(j - base) & (SPAN - 1);
        if (!(bits[b >> 5] >> (b & 31) & 1)) rest += exp2_64<7>(weight.log2_of(z));
    });
    rest = block_sum<THREADS>(rest, part_d);
    if (threadIdx.x == 0) out[blockIdx.x] = PartSums{rest, m, 0.0f};
}

template <typename T>
__global__ __launch_bounds__(THREADS) void distill_row_kernel(DistillArgs a, int row0, int parts, const PartSums *in, RowSums *out) {
    __shared__ uint32_t bits[LIST_BITS / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    __shared__ float part_f[2][THREADS / 64];
    __shared__ double part_d[4][THREADS / 64];
    constexpr int OWN = LOGITS_MAX_TOP / THREADS;
    const long r = (long)row0 + blockIdx.x;
    const int n = a.in.n;
    uint32_t mask = 31;
    while ((int)mask + 1 < n && mask + 1 < LIST_BITS) mask = mask * 2 + 1;
    mark_list(a, r, 0, n, mask, bits, list, &twice);
    in += (long)blockIdx.x * parts;
    auto larger = [](float x, float y) { return x != x || y != y ? NAN : fmaxf(x, y); };
    float m = -INFINITY, tm = -INFINITY;
    for (int p = threadIdx.x; p < parts; p += THREADS) m = larger(m, in[p].best);
    bool counts[OWN];
    float t[OWN], z[OWN];
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int i = o * THREADS + threadIdx.x;
        counts[o] = i < a.k && entry_counts(list, i, 0, n, twice);
        t[o] = counts[o] ? a.values[r * a.k + i] : -INFINITY;
        z[o] = counts[o] ? logit<T>(a, r, list[i]) : -INFINITY;
        tm = larger(tm, t[o]);
    }
    m = block_all<THREADS>(m, part_f[0], larger);
    tm = block_all<THREADS>(tm, part_f[1], larger);
    const double inv_t = 1.0 / (double)a.temperature;
    const Weight student(m, inv_t), teacher(tm, inv_t);
    double rest = 0.0, sum = 0.0, list_sum = 0.0;
    for (int p = threadIdx.x; p < parts; p += THREADS)
        if (in[p].rest != 0.0) rest += in[p].rest * exp2_64<11>(student.log2_of(in[p].best));
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (counts[o]) sum += exp2_64<11>(student.log2_of(z[o])), list_sum += exp2_64<11>(teacher.log2_of(t[o]));
    rest = block_sum<THREADS>(rest, part_d[0]);
    sum = rest + block_sum<THREADS>(sum, part_d[1]);
    list_sum = block_sum<THREADS>(list_sum, part_d[2]);
    const bool nan = m != m || tm != tm;
    double mass = a.rest ? (double)a.rest[r] : 0.0;  // outside the list
    mass = mass < 0.0 ? 0.0 : mass > 1.0 ? 1.0 : mass;
    const bool empty = !nan && (m == -INFINITY || tm == -INFINITY);
    constexpr double LN2 = 6.931471805599453094e-01;
    double loss = 0.0;
    const double log_sum = log(sum), log_list = log1p(-mass) - log(list_sum);
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (counts[o]) {
            const double log_p = teacher.log2_of(t[o]) * LN2 + log_list;
            const double p = exp(log_p);
            if (p != 0.0) loss += p * (log_p - (student.log2_of(z[o]) * LN2 - log_sum));
        }
    loss = block_sum<THREADS>(loss, part_d[3]);
    if (threadIdx.x == 0) {
        if (mass != 0.0) loss += mass * (log(mass) - (log(rest) - log_sum));
        if (a.loss) a.loss[r] = empty ? 0.0f : nan ? NAN : (float)loss;
        const float w = empty ? 0.0f : a.weight ? a.weight[r] : 1.0f;
        const double share = mass == 0.0 ? 1.0 / sum : rest > 0.0 ? 1.0 / sum - mass / rest : 0.0;
        out[blockIdx.x] = RowSums{nan ? NAN : 1.0 / sum, (1.0 - mass) / list_sum, nan ? NAN : w * inv_t * share, m, tm, (float)(w * inv_t), 0.0f};
    }
}

template <typename T>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(DistillArgs a, int row0, int parts, const RowSums *in) {
    constexpr int PER = 16 / sizeof(T), SPAN = PART_PIECES * PER, OWN = LOGITS_MAX_TOP / THREADS;
    __shared__ uint32_t bits[SPAN / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    const long r = (long)row0 + blockIdx.x / parts;
    const int part = blockIdx.x % parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Row<T> row(a.in, r, wave, THREADS / 64, lane, part * PART_PIECES, PART_PIECES);
    const int low = max(first_index(part, PER, row.lead), 0), high = min(first_index(part + 1, PER, row.lead), a.in.n);
    const RowSums sums = in[blockIdx.x / parts];
    T *grad = static_cast<T *>(a.grad) + r * a.grad_stride;
    const bool zero = sums.weight == 0.0f;
    mark_list(a, r, low, high, SPAN - 1, bits, list, &twice);
    // the listed classes' own terms, before anything is written (the gradient may take the logits' place)
    float own[OWN];
    bool counts[OWN];
    const double inv_t = 1.0 / (double)a.temperature;
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int i = o * THREADS + threadIdx.x;
        counts[o] = i < a.k && entry_counts(list, i, low, high, twice);
        own[o] = 0.0f;
        if (counts[o] && !zero) {
            const double e = exp2_64<11>(Weight(sums.best, inv_t).log2_of(logit<T>(a, r, list[i])));
            const double p = exp2_64<11>(Weight(sums.list_best, inv_t).log2_of(a.values[r * a.k + i])) * sums.list_scale;
            own[o] = (float)((e * sums.inv_sum - p) * (double)sums.weight);
        }
    }
    __syncthreads();
    const Weight weight(sums.best, inv_t);
    const bool together = ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(row.x)) & 15) == 0;
    for (int i = 0; i < row.rounds; ++i) {
        const int j = row.index(i);
        float v[PER];
        unpack<T>(row.load(i), v);
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = zero ? 0.0f : (float)(exp2_64<7>(weight.log2_of(v[e])) * sums.rest_scale);
        if (together && j >= 0 && j + PER <= a.in.n) {
            *reinterpret_cast<uint4 *>(grad + j) = pack<T>(v);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (j + e >= 0 && j + e < a.in.n) st1(grad + j + e, v[e]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (counts[o]) st1(grad + list[o * THREADS + threadIdx.x], own[o]);
}

// (for both types alike: the workspace's size does not depend on it, and float32 has more parts)
int rows_of_slice(int rows, int n) { return (int)std::min<long>(LOGITS_SLICE / logits_parts(n, false), rows); }

template <typename T>
hipError_t launch(const DistillArgs &a, char *ws, hipStream_t s) {
    const int parts = logits_parts(a.in.n, a.in.bf16);
    const int most = rows_of_slice(a.in.rows, a.in.n);
    RowSums *rows = reinterpret_cast<RowSums *>(ws);
    PartSums *sums = reinterpret_cast<PartSums *>(ws + most * sizeof(RowSums));
    for (long first = 0; first < a.in.rows; first += most) {
        const int r = (int)first, n = (int)std::min<long>(a.in.rows - first, most);
        distill_part_kernel<T><<<n * parts, THREADS, 0, s>>>(a, r, parts, sums);
        distill_row_kernel<T><<<n, THREADS, 0, s>>>(a, r, parts, sums, rows);
        if (a.grad) distill_grad_kernel<T><<<n * parts, THREADS, 0, s>>>(a, r, parts, rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t logits_workspace_bytes(int rows, int n) {
    return rows_of_slice(rows, n) * (sizeof(RowSums) + logits_parts(n, false) * sizeof(PartSums));
}

hipError_t launch_distill(const DistillArgs &a, void *ws, hipStream_t s) {
    return a.in.bf16 ? launch<uint16_t>(a, static_cast<char *>(ws), s) : launch<float>(a, static_cast<char *>(ws), s);
}

}  // namespace sushi
