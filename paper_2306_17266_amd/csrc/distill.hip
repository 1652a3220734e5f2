// Distillation from a teacher's leading logits (logits.h): the loss of a row and its gradient.
//
//   q = softmax(z / T);  e_j = exp((z_j - max z) / T), S = their sum
//   for the classes that are not listed, u = the largest of their logits:  f_j = exp((z_j - u) / T), R = their sum, A = exp((u - max z) / T)
//   p_i = (1 - r) softmax(t / T) over the row's list, r = the mass outside it
//   loss  = sum_i p_i (ln p_i - ln q_i) + r (ln r - (u - max z) / T - ln R + ln S)
//   d loss / d z_j = (e_j / S - p_j) / T for a listed class, f_j (A / S - r / R) / T for another
//
// The loss is a small difference of large terms where student and teacher agree: the unlisted weights are summed by themselves, never
// as S minus the list, and the sums, the list's terms and the logarithms have 64 bits.  Where the student is sure of its list, A passes
// below 2^-1074 (a gap of 745 T) while its logarithm and R, which is at least 1, are ordinary numbers.
#include <algorithm>

#include "logits_device.h"

namespace sushi {

namespace {

constexpr int THREADS = 256;
constexpr int LIST_BITS = 1 << 18;
constexpr double LN2 = 6.931471805599453094e-01;

// What a part of a row adds to it, and what a row's loss and gradient need, in the workspace.
struct PartSums {
    double rest;  // sum of the weights of what is not listed, relative to the largest of them in the part
    float best;   // that logit; NaN if there is one among them
    float pad;
};
struct RowSums {
    double inv_sum;     // 1 / S
    double list_scale;  // (1 - r) / sum of exp((t - max t) / T)
    double rest_scale;  // weight (A / S - r / R) / T
    double weight;      // divided by T; 0: the gradient is zero
    float best, list_best;
    float rest_best;  // u, read as the row is (as_infinite)
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

__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }  // (NaN if one is)

// The maximum of this thread's logits, NaN if there is one among them.
template <typename R>
__device__ __forceinline__ float own_largest(const R &row) {
    float m = -INFINITY;
    row.each([&](float z, int) { m = larger(m, z); });
    return m;
}

// Takes the listed classes out of a row in registers (they read as -inf): their terms are summed apart.  origin: index of bit 0.
template <typename T, int N>
__device__ __forceinline__ void leave_unlisted(HeldRow<T, N> &row, const uint32_t *bits, int origin) {
    constexpr int PER = HeldRow<T, N>::PER;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int b = row.index(i) - origin;  // (a multiple of PER)
        const uint32_t marks = i < row.rounds ? bits[b >> 5] >> (b & 31) & ((1u << PER) - 1) : 0;
        if (marks) {
            float v[PER];
            unpack<T>(row.raw[i], v);
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = marks >> e & 1 ? -INFINITY : v[e];
            row.raw[i] = pack<T>(v);
        }
    }
}

// Weights of listed classes, one at a time.
struct Terms : Weight {
    bool infinite;
    __device__ __forceinline__ Terms(float m, double inv_t) : Weight(m == INFINITY ? 0.0f : m, inv_t), infinite(m == INFINITY) {}
    __device__ __forceinline__ double log2_of(float z) const { return Weight::log2_of(infinite ? as_infinite(z) : z); }
};

// What belongs to a row besides its logits and its list; loaded before it is needed.
struct RowInputs {
    float rest, weight;
    __device__ __forceinline__ RowInputs(const DistillArgs &a, long r) {
        const float *any = reinterpret_cast<const float *>(a.classes);  // (without a branch for each)
        rest = (a.rest ? a.rest : any)[r], weight = (a.weight ? a.weight : any)[r];
        rest = a.rest ? rest : 0.0f, weight = a.weight ? weight : 1.0f;
    }
};

// This thread's entries of a row's list.
template <int OWN>
struct Entries {
    bool counts[OWN];
    float t[OWN], z[OWN];
};
template <typename T, int THREADS, int OWN>
__device__ __forceinline__ Entries<OWN> read_entries(const DistillArgs &a, long r, const int *list, int twice) {
    Entries<OWN> own;
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int i = o * THREADS + threadIdx.x;
        own.counts[o] = i < a.k && entry_counts(list, i, 0, a.in.n, twice);
        own.t[o] = own.counts[o] ? a.values[r * a.k + i] : -INFINITY;
        own.z[o] = own.counts[o] ? ld1(static_cast<const T *>(a.in.x) + r * a.in.stride + list[i]) : -INFINITY;
    }
    return own;
}

// The maxima of a row, of its unlisted logits, of the teacher's list.
struct Maxima {
    float row, rest, list;
    // u, where the row is read as as_infinite() says if its maximum is infinite
    __device__ __forceinline__ float anchor() const { return row == INFINITY ? as_infinite(rest) : rest; }
};
// m: of this thread's unlisted logits.  Only the waves that have entries look at them.
template <int THREADS, int OWN>
__device__ __forceinline__ Maxima maxima(float m, int k, const Entries<OWN> &own, float (*part)[THREADS / 64]) {
    float z = -INFINITY, t = -INFINITY;
    if ((int)(threadIdx.x & ~63u) < k) {
#pragma unroll
        for (int o = 0; o < OWN; ++o) z = larger(z, own.z[o]), t = larger(t, own.t[o]);
        z = wave_all(z, larger), t = wave_all(t, larger);
    }
    m = wave_all(m, larger);
    if ((threadIdx.x & 63) == 0) part[0][threadIdx.x >> 6] = m, part[1][threadIdx.x >> 6] = z, part[2][threadIdx.x >> 6] = t;
    __syncthreads();
    m = across_waves<THREADS / 64>(part[0], larger);
    return Maxima{larger(m, across_waves<THREADS / 64>(part[1], larger)), m, across_waves<THREADS / 64>(part[2], larger)};
}

// The row's loss (written) and what its gradient needs, from the maxima and each thread's part of R.  Only the waves that have
// entries compute with them.
template <int THREADS, int OWN>
__device__ __forceinline__ RowSums finish_row(const DistillArgs &a, long r, const RowInputs &row, const Maxima &top, double rest, const Entries<OWN> &own, double (*part)[THREADS / 64]) {
    const int wave = threadIdx.x >> 6;
    const bool entries = wave * 64 < a.k;
    const double inv_t = 1.0 / (double)a.temperature;
    const Terms student(top.row, inv_t), teacher(top.list, inv_t);
    double sum = 0.0, list_sum = 0.0;
    if (entries) {
#pragma unroll
        for (int o = 0; o < OWN; ++o)
            if (own.counts[o]) sum += exp2_64<11>(student.log2_of(own.z[o])), list_sum += exp2_64<11>(teacher.log2_of(own.t[o]));
        sum = wave_sum(sum), list_sum = wave_sum(list_sum);
    }
    rest = wave_sum(rest);
    if ((threadIdx.x & 63) == 0) part[0][wave] = rest, part[1][wave] = sum, part[2][wave] = list_sum;
    __syncthreads();
    const double log2_u = student.log2_of(top.rest), a_u = exp2_64<11>(log2_u);  // of A, A
    rest = sum_across<THREADS / 64>(part[0]), list_sum = sum_across<THREADS / 64>(part[2]);
    sum = rest * a_u + sum_across<THREADS / 64>(part[1]);
    const bool nan = top.row != top.row || top.list != top.list;
    double mass = row.rest;  // outside the list
    mass = mass < 0.0 ? 0.0 : mass > 1.0 ? 1.0 : mass;
    const bool empty = !nan && (top.row == -INFINITY || top.list == -INFINITY);
    if (a.loss) {
        double loss = 0.0;
        if (entries) {
            const double log_sum = log2_64(sum) * LN2, log_list = (log2_64(1.0 - mass) - log2_64(list_sum)) * LN2;
#pragma unroll
            for (int o = 0; o < OWN; ++o)
                if (own.counts[o]) {
                    const double log_p = teacher.log2_of(own.t[o]) * LN2 + log_list;
                    const double p = exp2_64<11>(log_p * 1.4426950408889634074);
                    // (p = 0 counts nothing; what makes log_p NaN shows in the maxima or in the mass)
                    if (p != 0.0) loss += p * (log_p - (student.log2_of(own.z[o]) * LN2 - log_sum));
                }
            loss = wave_sum(loss);
            if (wave == 0 && mass != 0.0) loss += mass * ((log2_64(mass) - log2_64(rest) - log2_u) * LN2 + log_sum);
        }
        if (a.k > 64) {
            if ((threadIdx.x & 63) == 0) part[3][wave] = loss;
            __syncthreads();
            loss = sum_across<THREADS / 64>(part[3]);
        }
        if (threadIdx.x == 0) a.loss[r] = empty ? 0.0f : nan ? NAN : (float)loss;
    }
    const float w = empty ? 0.0f : row.weight;
    const double inv_sum = 1.0 / sum, share = mass == 0.0 ? a_u * inv_sum : rest > 0.0 ? a_u * inv_sum - mass / rest : 0.0, scale = w * inv_t * share;
    return RowSums{nan ? NAN : inv_sum, (1.0 - mass) / list_sum, nan || scale != scale ? NAN : scale, w * inv_t, top.row, top.list, top.anchor(), 0.0f};
}

// Gradient of a listed class.
__device__ __forceinline__ float list_gradient(const RowSums &s, double inv_t, float z, float t) {
    const double e = exp2_64<11>(Terms(s.best, inv_t).log2_of(z)), p = exp2_64<11>(Terms(s.list_best, inv_t).log2_of(t)) * s.list_scale;
    return (float)((e * s.inv_sum - p) * s.weight);
}

// Gradients of the others, out * 2^((z - u) * scale).  Weights have 32 bits here: what a gradient of 32 bits is left with is the
// rounding of the exponent, 2^-24 of it thrice, and what is 2^-126 of the row's largest is zero.
struct GradientOf {
    float best, scale, out;
    __device__ __forceinline__ GradientOf(const RowSums &s, double inv_t) {
        const bool zero = s.weight == 0.0;
        const double largest = 3.4028234663852886e38;  // (an infinite factor would make NaN of weights of zero)
        best = s.rest_best == -INFINITY || zero ? 0.0f : s.rest_best;  // (-inf: there are no others above it, and they get 0)
        scale = (float)fmin(1.4426950408889634074 * inv_t, largest);
        const double o = zero ? 0.0 : s.rest_scale;
        out = o != o ? NAN : (float)fmin(fmax(o, -largest), largest);
    }
    __device__ __forceinline__ float of(float z) const { return __builtin_amdgcn_exp2f((z - best) * scale) * out; }
};

// The elements of piece r (first index j) that are in the row, one by one.
template <typename T>
__device__ __forceinline__ void store_elements(T *grad, int n, int j, uint4 r) {
#pragma unroll 1
    for (int e = 0; e < 16 / (int)sizeof(T); ++e)
        if (j + e >= 0 && j + e < n) st1(grad + j + e, element<T>(r, e));
}

// ------------------------------------------------------------------ a row in the registers of a workgroup

// For gradients whose rows lie to 16 bytes as those of the logits do.  The logits stay in registers as they came, and their weights are
// computed again for the gradient: with 80 registers three workgroups of 512 share a compute unit, and one loads or stores while
// another computes.  4096 x 32000 in bf16, loss and gradient: 142 us, 542 MB at 3.8 TB/s (a copy reaches 5.1: floor 103); with two
// workgroups a compute unit 147, with four 152 (spilled registers), weights kept from the loss for the gradient 199 against 154 then.
// What is left is the loss: 25 instructions a logit that only partly run beside the loads and stores of other workgroups.
template <typename T, int N, int THREADS>
__global__ __launch_bounds__(THREADS, 6) void distill_held_kernel(DistillArgs a, int row0) {
    constexpr int PER = 16 / sizeof(T), SPAN = N * THREADS * PER, OWN = (LOGITS_MAX_TOP + THREADS - 1) / THREADS;
    __shared__ uint32_t bits[SPAN / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    __shared__ float part_f[3][THREADS / 64];
    __shared__ double part_d[4][THREADS / 64];
    const long r = (long)row0 + blockIdx.x;
    HeldRow<T, N> row(a.in, r, threadIdx.x >> 6, THREADS / 64, threadIdx.x & 63);
    const RowInputs inputs(a, r);
    mark_list<THREADS>(a, r, 0, a.in.n, -row.lead, SPAN - 1, bits, list, &twice);
    const Entries<OWN> own = read_entries<T, THREADS, OWN>(a, r, list, twice);
    leave_unlisted(row, bits, -row.lead);
    const Maxima top = maxima<THREADS>(own_largest(row), a.k, own, part_f);
    const double inv_t = 1.0 / (double)a.temperature;
    if (top.row == INFINITY) row.only_infinite();
    const Weight weight(top.anchor(), inv_t);
    double rest = 0.0;
    row.each([&](float z, int) { rest += exp2_64<6>(weight.log2_of(z)); });
    const RowSums s = finish_row<THREADS>(a, r, inputs, top, rest, own, part_d);
    if (!a.grad) return;
    // (the gradient may take the logits' place: every thread has passed a barrier since its logits were read)
    T *grad = static_cast<T *>(a.grad) + r * a.grad_stride;
    const bool zero = s.weight == 0.0;
    if (zero) row.none();
    const GradientOf gradient(s, inv_t);
    T *piece = grad + row.index(0);
    uint4 start = row.raw[0], end = row.raw[0];
    const int i_end = row.partial_end();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < row.rounds) {
            float v[PER];
            unpack<T>(row.raw[i], v);
#pragma unroll
            for (int e = 0; e < PER; ++e) v[e] = gradient.of(v[e]);
            const uint4 g = pack<T>(v);
            const int j = row.index(i);
            if (j >= 0 && j + PER <= a.in.n) *reinterpret_cast<uint4 *>(piece + i * 64 * PER) = g;
            if (i == 0) start = g;
            end = choose(i == i_end, g, end);
            apart();
        }
    if (row.index(0) < 0 && row.index(0) + PER > 0) store_elements(grad, a.in.n, row.index(0), start);
    if (i_end >= 0) store_elements(grad, a.in.n, row.index(i_end), end);
    __syncthreads();
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (own.counts[o]) st1(grad + list[o * THREADS + threadIdx.x], zero ? 0.0f : list_gradient(s, inv_t, own.z[o], own.t[o]));
}

// ------------------------------------------------------------------ a row in parts

// 5 x 250007 in bf16, loss: 10.7 us; 4.8 for the parts and 7 for what a row's workgroup does with its list and sums, one wait
// after another.
template <typename T, int PIECES>
__global__ __launch_bounds__(THREADS) void distill_part_kernel(DistillArgs a, int row0, int parts, PartSums *out) {
    constexpr int PER = 16 / sizeof(T), SPAN = PIECES * PER;
    __shared__ uint32_t bits[SPAN / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    __shared__ float part_f[THREADS / 64];
    __shared__ double part_d[THREADS / 64];
    const long r = (long)row0 + blockIdx.x / parts;
    const int part = blockIdx.x % parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    HeldRow<T, PIECES / THREADS> row(a.in, r, wave, THREADS / 64, lane, part * PIECES, PIECES);
    const int origin = part * SPAN - row.lead;
    mark_list<THREADS>(a, r, max(origin, 0), min(origin + SPAN, a.in.n), origin, SPAN - 1, bits, list, &twice);
    leave_unlisted(row, bits, origin);
    const float m = block_all<THREADS>(own_largest(row), part_f, larger);
    if (m == INFINITY) row.only_infinite();
    const Weight weight(m == INFINITY ? 0.0f : m, 1.0 / (double)a.temperature);
    double rest = 0.0;
    row.each([&](float z, int) { rest += exp2_64<6>(weight.log2_of(z)); });
    rest = block_sum<THREADS>(rest, part_d);
    if (threadIdx.x == 0) out[blockIdx.x] = PartSums{rest, m, 0.0f};
}

// Rows of more than LIST_BITS classes share marks: with 1024 of 2^20 classes one or two pairs usually do, and each entry is then compared with
// those before it (4 x 1048576, loss: 181 us with 1024 entries, 13 with 64; 4 x 262144 with 1024: 12).
template <typename T>
__global__ __launch_bounds__(THREADS) void distill_row_kernel(DistillArgs a, int row0, int parts, const PartSums *in, RowSums *out) {
    __shared__ uint32_t bits[LIST_BITS / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    __shared__ float part_f[3][THREADS / 64];
    __shared__ double part_d[4][THREADS / 64];
    constexpr int OWN = LOGITS_MAX_TOP / THREADS;
    const long r = (long)row0 + blockIdx.x;
    const int n = a.in.n;
    const RowInputs inputs(a, r);
    uint32_t mask = 31;
    while ((int)mask + 1 < n && mask + 1 < LIST_BITS) mask = mask * 2 + 1;
    mark_list<THREADS>(a, r, 0, n, 0, mask, bits, list, &twice);
    in += (long)blockIdx.x * parts;
    const Entries<OWN> own = read_entries<T, THREADS, OWN>(a, r, list, twice);
    float m = -INFINITY;
    for (int p = threadIdx.x; p < parts; p += THREADS) m = larger(m, in[p].best);
    const Maxima top = maxima<THREADS>(m, a.k, own, part_f);
    const Weight weight(top.anchor(), 1.0 / (double)a.temperature);
    double rest = 0.0;
    for (int p = threadIdx.x; p < parts; p += THREADS)
        if (in[p].rest != 0.0) rest += in[p].rest * exp2_64<11>(weight.log2_of(top.row == INFINITY ? as_infinite(in[p].best) : in[p].best));
    const RowSums s = finish_row<THREADS>(a, r, inputs, top, rest, own, part_d);
    if (threadIdx.x == 0) out[blockIdx.x] = s;
}

template <typename T, int PIECES>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(DistillArgs a, int row0, int parts, const RowSums *in) {
    constexpr int PER = 16 / sizeof(T), SPAN = PIECES * PER, OWN = LOGITS_MAX_TOP / THREADS;
    __shared__ uint32_t bits[SPAN / 32];
    __shared__ int list[LOGITS_MAX_TOP];
    __shared__ int twice;
    const long r = (long)row0 + blockIdx.x / parts;
    const int part = blockIdx.x % parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Row<T> row(a.in, r, wave, THREADS / 64, lane, part * PIECES, PIECES);
    const int origin = part * SPAN - row.lead, low = max(origin, 0), high = min(origin + SPAN, a.in.n);
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
        if (counts[o] && s.weight != 0.0) own[o] = list_gradient(s, 1.0 / (double)a.temperature, ld1(row.x + list[i]), a.values[r * a.k + i]);
    }
    __syncthreads();
    if (s.best == INFINITY) row.only_infinite();
    const bool together = ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(row.x)) & 15) == 0, zero = s.weight == 0.0;
    const GradientOf gradient(s, 1.0 / (double)a.temperature);
    for (int i = 0; i < row.rounds; ++i) {
        float v[PER];
        unpack<T>(row.load(i), v);
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = zero ? 0.0f : gradient.of(v[e]);
        const int j = row.index(i);
        if (together && j >= 0 && j + PER <= a.in.n)
            *reinterpret_cast<uint4 *>(grad + j) = pack<T>(v);
        else
            store_elements(grad, a.in.n, j, pack<T>(v));
    }
    __syncthreads();
#pragma unroll
    for (int o = 0; o < OWN; ++o)
        if (counts[o]) st1(grad + list[o * THREADS + threadIdx.x], own[o]);
}

template <typename T, int N, int HELD>
hipError_t launch_held(const DistillArgs &a, hipStream_t s) {
    const long most = (1l << 31) / HELD;
    for (long first = 0; first < a.in.rows; first += most) {
        const int n = (int)std::min<long>(a.in.rows - first, most);
        distill_held_kernel<T, N, HELD><<<n, HELD, 0, s>>>(a, (int)first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// most: rows of a launch.
template <typename T, int PIECES>
hipError_t launch_parts(const DistillArgs &a, int pieces, long most, char *ws, hipStream_t s) {
    const int parts = logits_parts(pieces, PIECES);
    RowSums *rows = reinterpret_cast<RowSums *>(ws);
    PartSums *sums = reinterpret_cast<PartSums *>(ws + most * sizeof(RowSums));
    for (long first = 0; first < a.in.rows; first += most) {
        const int r = (int)first, n = (int)std::min<long>(a.in.rows - first, most);
        distill_part_kernel<T, PIECES><<<n * parts, THREADS, 0, s>>>(a, r, parts, sums);
        distill_row_kernel<T><<<n, THREADS, 0, s>>>(a, r, parts, sums, rows);
        if (a.grad) distill_grad_kernel<T, PIECES><<<n * parts, THREADS, 0, s>>>(a, r, parts, rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t launch(const DistillArgs &a, char *ws, hipStream_t s) {
    const int pieces = logits_pieces(a.in.n, a.in.bf16);
    // Gradients whose rows lie otherwise within 16 bytes are stored an element at a time, in parts: 256 x 1000 in float32 14 us against
    // 8.5, 4096 x 32000 in bf16 313 against 155.
    const bool together = !a.grad || ((reinterpret_cast<uintptr_t>(a.grad) - reinterpret_cast<uintptr_t>(a.in.x)) % 16 == 0 &&
                                      (a.in.rows == 1 || (a.grad_stride - a.in.stride) * (long)sizeof(T) % 16 == 0));
    if (together && held_rows(a.in)) {
        if (pieces <= 256) return launch_held<T, 1, 256>(a, s);
        if (pieces <= 1024) return launch_held<T, 4, 256>(a, s);
        if (pieces <= 4096) return launch_held<T, 8, 512>(a, s);
        return launch_held<T, 8, 1024>(a, s);
    }
    return small_parts(a.in, LOGITS_MOST_PARTS) ? launch_parts<T, LOGITS_SMALL_PART_PIECES>(a, pieces, a.in.rows, ws, s)
                             : launch_parts<T, LOGITS_PART_PIECES>(a, pieces, std::min<long>(rows_of_slice(a.in.n), a.in.rows), ws, s);
}

}  // namespace

size_t distill_part_bytes() { return sizeof(PartSums); }
size_t distill_row_bytes() { return sizeof(RowSums); }

size_t logits_workspace_bytes(int rows, int n) {
    const int pieces = logits_pieces(n, false);
    const size_t slice = std::min<long>(rows_of_slice(n), rows), parts = slice * logits_parts(pieces, LOGITS_PART_PIECES);
    const size_t few = std::min(rows, LOGITS_MOST_SMALL_PARTS), small = std::min<size_t>(few * logits_parts(pieces, LOGITS_SMALL_PART_PIECES), LOGITS_MOST_SMALL_PARTS);
    const size_t distill = std::max(parts, small) * distill_part_bytes() + std::max(slice, few) * distill_row_bytes();
    if (n <= LOGITS_HELD_PLAIN_FEW) return distill;  // (the others hold these rows, of either type)
    return std::max({distill,
                     std::max(parts, small) * sample_part_bytes() + std::max(slice, few) * sample_row_bytes(), parts * top_logits_part_bytes()});
}

hipError_t launch_distill(const DistillArgs &a, void *ws, hipStream_t s) {
    return a.in.bf16 ? launch<uint16_t>(a, static_cast<char *>(ws), s) : launch<float>(a, static_cast<char *>(ws), s);
}

}  // namespace sushi
