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
constexpr double LN2 = 6.931471805599453094e-01;

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

// The row's list in LDS, with a mark for every class in [low, high): bit (class - origin) & mask.  Returns with *twice set if a class may
// stand there twice.  Entries outside are none of this workgroup's business.
template <int THREADS>
__device__ __forceinline__ void mark_list(const DistillArgs &a, long r, int low, int high, int origin, uint32_t mask, uint32_t *bits, int *list, int *twice) {
    for (uint32_t w = threadIdx.x; w <= mask >> 5; w += THREADS) bits[w] = 0;
    if (threadIdx.x == 0) *twice = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.k; i += THREADS) {
        const int c = a.classes[r * a.k + i];
        list[i] = c;
        if (c >= low && c < high) {
            const uint32_t b = (uint32_t)(c - origin) & mask;
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

// Marks of a piece whose first element is at bit b (a multiple of its length).
template <typename T>
__device__ __forceinline__ uint32_t piece_marks(const uint32_t *bits, int b) {
    return bits[b >> 5] >> (b & 31);
}

__device__ __forceinline__ float larger(float x, float y) { return x != x || y != y ? NAN : fmaxf(x, y); }

// The maximum of a row or part, NaN if there is one, and its share of R at a maximum.
template <int THREADS, typename R>
__device__ __forceinline__ float largest(const R &row, float *part) {
    float m = -INFINITY;
    bool nan = false;
    row.each([&](float z, int) { m = fmaxf(m, z), nan |= z != z; });
    return block_all<THREADS>(nan ? NAN : m, part, larger);
}
template <typename T, typename R>
__device__ __forceinline__ double sum_unlisted(const R &row, const Weight &weight, const uint32_t *bits, int origin) {
    double rest = 0.0;
    row.each_piece([&](const float(&v)[R::PER], int j) {
        const uint32_t marks = piece_marks<T>(bits, j - origin);
#pragma unroll
        for (int e = 0; e < R::PER; ++e) {
            const double w = exp2_64<7>(weight.log2_of(v[e]));
            rest += marks >> e & 1 ? 0.0 : w;
        }
    });
    return rest;
}

// This thread's entries of a row's list.
template <int OWN>
struct Entries {
    bool counts[OWN];
    float t[OWN], z[OWN];
};

// The row's loss (written) and what its gradient needs, from its maximum m and R, which every thread has.
template <typename T, int THREADS, int OWN>
__device__ __forceinline__ RowSums finish_row(const DistillArgs &a, long r, float m, double rest, const Entries<OWN> &own, float *part_f, double (*part_d)[THREADS / 64]) {
    float tm = -INFINITY;
#pragma unroll
    for (int o = 0; o < OWN; ++o) tm = larger(tm, own.t[o]);
    tm = block_all<THREADS>(tm, part_f, larger);
    const double inv_t = 1.0 / (double)a.temperature;
    const Weight student(m, inv_t), teacher(tm, inv_t);
    double sum = 0.0, list_sum = 0.0;
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (own.counts[o]) sum += exp2_64<11>(student.log2_of(own.z[o])), list_sum += exp2_64<11>(teacher.log2_of(own.t[o]));
    sum = wave_sum(sum), list_sum = wave_sum(list_sum);
    if ((threadIdx.x & 63) == 0) part_d[0][threadIdx.x >> 6] = sum, part_d[1][threadIdx.x >> 6] = list_sum;
    __syncthreads();
    sum = rest, list_sum = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) sum += part_d[0][w], list_sum += part_d[1][w];
    const bool nan = m != m || tm != tm;
    double mass = a.rest ? (double)a.rest[r] : 0.0;  // outside the list
    mass = mass < 0.0 ? 0.0 : mass > 1.0 ? 1.0 : mass;
    const bool empty = !nan && (m == -INFINITY || tm == -INFINITY);
    if (a.loss) {
        double loss = 0.0;
        const double log_sum = log(sum), log_list = log1p(-mass) - log(list_sum);
#pragma unroll
        for (int o = 0; o < OWN; ++o)
            if (own.counts[o]) {
                const double log_p = teacher.log2_of(own.t[o]) * LN2 + log_list;
                const double p = exp(log_p);
                if (p != 0.0) loss += p * (log_p - (student.log2_of(own.z[o]) * LN2 - log_sum));
            }
        loss = block_sum<THREADS>(loss, part_d[2]);
        if (threadIdx.x == 0) {
            if (mass != 0.0) loss += mass * (log(mass) - (log(rest) - log_sum));
            a.loss[r] = empty ? 0.0f : nan ? NAN : (float)loss;
        }
    }
    const float w = empty ? 0.0f : a.weight ? a.weight[r] : 1.0f;
    const double share = mass == 0.0 ? 1.0 / sum : rest > 0.0 ? 1.0 / sum - mass / rest : 0.0;
    return RowSums{nan ? NAN : 1.0 / sum, (1.0 - mass) / list_sum, nan ? NAN : w * inv_t * share, m, tm, (float)(w * inv_t), 0.0f};
}

// Gradient of a listed class.
__device__ __forceinline__ float list_gradient(const RowSums &s, double inv_t, float z, float t) {
    const double e = exp2_64<11>(Weight(s.best, inv_t).log2_of(z)), p = exp2_64<11>(Weight(s.list_best, inv_t).log2_of(t)) * s.list_scale;
    return (float)((e * s.inv_sum - p) * (double)s.weight);
}

// Gradient of every class of a row or part as if it were not listed.  The weights have 32 bits here: what a gradient of 32 bits is left
// with is the rounding of the exponent, 2^-24 of it thrice.
template <typename T, typename R>
__device__ __forceinline__ void write_gradient(const DistillArgs &a, const R &row, T *grad, const RowSums &s) {
    constexpr int PER = R::PER;
    const double inv_t = 1.0 / (double)a.temperature;
    const bool together = ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(row.x)) & 15) == 0;
    const bool zero = s.weight == 0.0f, infinite = s.best == INFINITY;
    const float scale = (float)(inv_t * 1.4426950408889634074), out = zero ? 0.0f : (float)s.rest_scale;
    row.each_piece([&](const float(&v)[PER], int j) {
        float g[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const float w = infinite ? (v[e] == INFINITY ? 1.0f : 0.0f) : __builtin_amdgcn_exp2f((v[e] - s.best) * scale);
            g[e] = zero ? 0.0f : w * out;
        }
        if (together && j >= 0 && j + PER <= a.in.n) {
            *reinterpret_cast<uint4 *>(grad + j) = pack<T>(g);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (j + e >= 0 && j + e < a.in.n) st1(grad + j + e, g[e]);
        }
    });
}

template <typename T>
__device__ __forceinline__ float logit(const DistillArgs &a, long r, int c) {
    return ld1(static_cast<const T *>(a.in.x) + r * a.in.stride + c);
}

// ------------------------------------------------------------------ a row in the registers of a workgroup

template <typename T, int N, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void distill_held_kernel(DistillArgs a, int row0) {
    constexpr int SPAN = N * THREADS * 16 / (int)sizeof(T), OWN = (LOGITS_MAX_TOP + THREADS - 1) / THREADS;
    __shared__ uint32_t bits[SPAN / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    __shared__ float part_f[2][THREADS / 64];
    __shared__ double part_d[4][THREADS / 64];
    const long r = (long)row0 + blockIdx.x;
    const HeldRow<T, N> row(a.in, r, threadIdx.x >> 6, THREADS / 64, threadIdx.x & 63);
    mark_list<THREADS>(a, r, 0, a.in.n, -row.lead, SPAN - 1, bits, list, &twice);
    Entries<OWN> own;
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int i = o * THREADS + threadIdx.x;
        own.counts[o] = i < a.k && entry_counts(list, i, 0, a.in.n, twice);
        own.t[o] = own.counts[o] ? a.values[r * a.k + i] : -INFINITY;
        own.z[o] = own.counts[o] ? logit<T>(a, r, list[i]) : -INFINITY;
    }
    const float m = largest<THREADS>(row, part_f[0]);
    const double inv_t = 1.0 / (double)a.temperature;
    const double rest = block_sum<THREADS>(sum_unlisted<T>(row, Weight(m, inv_t), bits, -row.lead), part_d[3]);
    const RowSums s = finish_row<T, THREADS>(a, r, m, rest, own, part_f[1], part_d);
    if (!a.grad) return;
    // (the gradient may take the logits' place: every thread has passed a barrier since its logits were read)
    T *grad = static_cast<T *>(a.grad) + r * a.grad_stride;
    write_gradient<T>(a, row, grad, s);
    __syncthreads();
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (own.counts[o]) st1(grad + list[o * THREADS + threadIdx.x], s.weight == 0.0f ? 0.0f : list_gradient(s, inv_t, own.z[o], own.t[o]));
}

// ------------------------------------------------------------------ a row in parts

__device__ __forceinline__ int first_index(int part, int per, int lead) { return part * PART_PIECES * per - lead; }

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
    const HeldRow<T, PART_PIECES / THREADS> row(a.in, r, wave, THREADS / 64, lane, part * PART_PIECES, PART_PIECES);
    const int origin = first_index(part, PER, row.lead);
    mark_list<THREADS>(a, r, max(origin, 0), min(origin + SPAN, a.in.n), origin, SPAN - 1, bits, list, &twice);
    const float m = largest<THREADS>(row, part_f);
    const double rest = block_sum<THREADS>(sum_unlisted<T>(row, Weight(m, 1.0 / (double)a.temperature), bits, origin), part_d);
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
    mark_list<THREADS>(a, r, 0, n, 0, mask, bits, list, &twice);
    in += (long)blockIdx.x * parts;
    float m = -INFINITY;
    for (int p = threadIdx.x; p < parts; p += THREADS) m = larger(m, in[p].best);
    Entries<OWN> own;
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int i = o * THREADS + threadIdx.x;
        own.counts[o] = i < a.k && entry_counts(list, i, 0, n, twice);
        own.t[o] = own.counts[o] ? a.values[r * a.k + i] : -INFINITY;
        own.z[o] = own.counts[o] ? logit<T>(a, r, list[i]) : -INFINITY;
    }
    m = block_all<THREADS>(m, part_f[0], larger);
    const Weight student(m, 1.0 / (double)a.temperature);
    double rest = 0.0;
    for (int p = threadIdx.x; p < parts; p += THREADS)
        if (in[p].rest != 0.0) rest += in[p].rest * exp2_64<11>(student.log2_of(in[p].best));
    rest = block_sum<THREADS>(rest, part_d[3]);
    const RowSums s = finish_row<T, THREADS>(a, r, m, rest, own, part_f[1], part_d);
    if (threadIdx.x == 0) out[blockIdx.x] = s;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(DistillArgs a, int row0, int parts, const RowSums *in) {
    constexpr int PER = 16 / sizeof(T), SPAN = PART_PIECES * PER, OWN = LOGITS_MAX_TOP / THREADS;
    __shared__ uint32_t bits[SPAN / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    const long r = (long)row0 + blockIdx.x / parts;
    const int part = blockIdx.x % parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const HeldRow<T, PART_PIECES / THREADS> row(a.in, r, wave, THREADS / 64, lane, part * PART_PIECES, PART_PIECES);
    const int origin = first_index(part, PER, row.lead), low = max(origin, 0), high = min(origin + SPAN, a.in.n);
    const RowSums s = in[blockIdx.x / parts];
    T *grad = static_cast<T *>(a.grad) + r * a.grad_stride;
    mark_list<THREADS>(a, r, low, high, origin, SPAN - 1, bits, list, &twice);
    // the listed classes' own terms, before anything is written (the gradient may take the logits' place)
    float own[OWN];
    bool counts[OWN];
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int i = o * THREADS + threadIdx.x;
        counts[o] = i < a.k && entry_counts(list, i, low, high, twice);
        own[o] = 0.0f;
        if (counts[o] && s.weight != 0.0f) own[o] = list_gradient(s, 1.0 / (double)a.temperature, logit<T>(a, r, list[i]), a.values[r * a.k + i]);
    }
    __syncthreads();
    write_gradient<T>(a, row, grad, s);
    __syncthreads();
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (counts[o]) st1(grad + list[o * THREADS + threadIdx.x], own[o]);
}

template <typename T, int N, int HELD>
hipError_t launch_held(const DistillArgs &a, hipStream_t s) {
    const long most = (1l << 31) / HELD;
    for (long first = 0; first < a.in.rows; first += most) {
        distill_held_kernel<T, N, HELD><<<(int)std::min<long>(a.in.rows - first, most), HELD, 0, s>>>(a, (int)first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// (for both types alike: the workspace's size does not depend on it, and float32 has more parts)
int rows_of_slice(int rows, int n) { return (int)std::min<long>(LOGITS_SLICE / logits_parts(n, false), rows); }

template <typename T>
hipError_t launch(const DistillArgs &a, char *ws, hipStream_t s) {
    constexpr int PER = 16 / sizeof(T);
    const int pieces = (a.in.n + 2 * PER - 2) / PER;  // (a row may start inside its first piece)
    if (pieces <= 256) return launch_held<T, 1, 256>(a, s);
    if (pieces <= 1024) return launch_held<T, 4, 256>(a, s);
    if (pieces <= 4096) return launch_held<T, 8, 512>(a, s);
    if (pieces <= 8192 && a.in.rows >= 256) return launch_held<T, 8, 1024>(a, s);
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
