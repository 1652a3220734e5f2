// Device-side helpers of the operators on logits: access to a row, weights, sums over waves and workgroups.
#pragma once

#include "device_common.h"
#include "logit_grid.h"
#include "logits.h"

namespace sushi {

// ------------------------------------------------------------------ weight of a logit (its order: logit_grid.h)

// 2^t for t <= 0 in 64 bits: t = i + f with |f| <= 1/2, a polynomial for 2^f, and i into the exponent.  Below 2^-1022, for -inf
// and for NaN: zero.  TERMS = 11: the power series, off by 2e-14 of the value at most.  TERMS = 6: for sums, off by 2e-9 at most; the
// coefficients come from a least-squares fit of the relative error, reweighted until its largest values were level, with 1 at f = 0.
template <int TERMS>
__device__ __forceinline__ double exp2_64(double t) {
    static_assert(TERMS == 6 || TERMS == 11, "one of the two polynomials");
    t = fmax(t, -1100.0);
    const double i = __builtin_rint(t), f = t - i;
    double p;
    if constexpr (TERMS == 6) {
        constexpr double c[6] = {0.6931472028559306, 0.24022647913391443, 0.05550332468951376, 0.009618437385012474, 0.0013398875357849087, 0.00015353355071142543};
        p = c[5];
#pragma unroll
        for (int n = 4; n >= 0; --n) p = fma(p, f, c[n]);
    } else {  // (ln 2)^n / n!
        constexpr double c[11] = {6.931471805599453094e-01, 2.402265069591007123e-01, 5.550410866482157995e-02, 9.618129107628477162e-03,
                                  1.333355814642844343e-03, 1.540353039338160995e-04, 1.525273380405984028e-05, 1.321548679014430949e-06,
                                  1.017808600923969973e-07, 7.054911620801123330e-09, 4.445538271870811498e-10};
        p = c[10];
#pragma unroll
        for (int n = 9; n >= 0; --n) p = fma(p, f, c[n]);
    }
    return ldexp(fma(p, f, 1.0), (int)i);
}

// log2 in 64 bits, off by 1e-13 at most: the 32-bit one, and what its result lacks by two terms of the series of log(1 + d).
__device__ __forceinline__ double log2_64(double x) {
    const double m = __builtin_amdgcn_frexp_mant(x);
    const float y = __builtin_amdgcn_logf((float)m);
    const double d = fma(m, exp2_64<11>(-(double)y), -1.0);
    const double r = (double)__builtin_amdgcn_frexp_exp(x) + ((double)y + d * fma(d, -0.5, 1.0) * 1.4426950408889634074);
    return x > 0.0 ? r : x == 0.0 ? -INFINITY : NAN;
}

// Weights of a row's logits at a temperature: 2^log2_of().  An infinite maximum is no case of its own here: its row is read as
// Row::only_infinite() says.
struct Weight {
    double best, scale;  // maximum; log2(e) / T
    __device__ __forceinline__ Weight(float m, double inv_t) : best(m), scale(inv_t * 1.4426950408889634074) {}
    __device__ __forceinline__ double log2_of(float z) const { return ((double)z - best) * scale; }  // <= 0, or NaN for what has no weight
};

// Where the maximum is +inf the weights have a limit: the infinite logits share the row.  The same weights as those of zeros among -inf.
__device__ __forceinline__ float as_infinite(float z) { return z == INFINITY ? 0.0f : -INFINITY; }

// ------------------------------------------------------------------ a row

template <typename T>
__device__ __forceinline__ void unpack(uint4 r, float (&v)[16 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
        v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y), v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
    } else {
        v[0] = bf2f(r.x & 0xFFFFu), v[1] = __uint_as_float(r.x & 0xFFFF0000u), v[2] = bf2f(r.y & 0xFFFFu), v[3] = __uint_as_float(r.y & 0xFFFF0000u);
        v[4] = bf2f(r.z & 0xFFFFu), v[5] = __uint_as_float(r.z & 0xFFFF0000u), v[6] = bf2f(r.w & 0xFFFFu), v[7] = __uint_as_float(r.w & 0xFFFF0000u);
    }
}

template <typename T>
__device__ __forceinline__ uint4 pack(const float (&v)[16 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else
        return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

template <typename T>
__device__ __forceinline__ uint4 share_infinite(uint4 r) {
    float v[16 / sizeof(T)];
    unpack<T>(r, v);
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) v[e] = as_infinite(v[e]);
    return pack<T>(v);
}

// Element e of a piece, e not known to the compiler (loops that run seldom stay small).
template <typename T>
__device__ __forceinline__ float element(uint4 r, int e) {
    const int w = sizeof(T) == 4 ? e : e >> 1;
    const uint32_t a = r.x, b = r.y, c = r.z, d = r.w;  // (a choice between the members themselves would be one between addresses)
    const uint32_t lo = w & 1 ? b : a, hi = w & 1 ? d : c, u = w & 2 ? hi : lo;
    if (sizeof(T) == 4) return __uint_as_float(u);
    return __uint_as_float(e & 1 ? u & 0xFFFF0000u : u << 16);
}

// f(logit, index) for the elements of a piece that are at least z_low.
template <typename T, typename F>
__device__ __forceinline__ void from_piece(uint4 r, int j, float z_low, F f) {
    float v[16 / sizeof(T)];
    unpack<T>(r, v);
    bool some = false;
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) some |= v[e] >= z_low;
    if (some) {
#pragma unroll 1
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) {
            const float z = element<T>(r, e);
            if (z >= z_low) f(z, j + e);
        }
    }
}

// One row, or a part of it, as a workgroup reads it: in pieces of 16 bytes at 16-byte addresses (the first and the last may be partly outside the
// row, whose start need not be aligned: what is outside is not loaded and reads as -inf).  Every wave has a run of pieces of
// its own, so that the order of (wave, round, lane, element) is the order of the indexes; neighbouring lanes have
// neighbouring pieces.
template <typename T>
struct Row {
    static constexpr int PER = 16 / sizeof(T);  // logits of a piece
    static constexpr uint32_t NONE = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;  // -inf
    const T *x;
    int n, lead;        // logits; elements of the first piece before the row
    int first, rounds;  // this lane's first piece, and how many it has (64 apart)
    bool infinite = false;

    // A part: `most` pieces, a multiple of 64 * waves, from piece `from` on.
    __device__ __forceinline__ Row(const LogitRows &in, long row, int wave, int waves, int lane, int from = 0, int most = 0x7FFFFFFF) {
        x = static_cast<const T *>(in.x) + row * in.stride;
        n = in.n;
        lead = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
        const int pieces = min((n + lead + PER - 1) / PER - from, most);
        rounds = pieces > 0 ? (pieces + 64 * waves - 1) / (64 * waves) : 0;
        first = from + wave * rounds * 64 + lane;
    }
    __device__ __forceinline__ int index(int i) const { return (first + i * 64) * PER - lead; }  // of the piece's first element
    // From here on the row reads as as_infinite() of its logits.
    __device__ __forceinline__ void only_infinite() { infinite = true; }
    __device__ __forceinline__ uint4 load(int i) const {
        uint4 r = load_plain(i);
        if (infinite) r = share_infinite<T>(r);
        return r;
    }
    __device__ __forceinline__ uint4 load_plain(int i) const {
        const int j = index(i);
        if (j >= 0 && j + PER <= n) return *reinterpret_cast<const uint4 *>(x + j);
        // (two elements of bf16 share a word, and each load waits for the one before: 256 x 999 takes 0.6 us more than 256 x 1000 in the
        // top logits and 1 in the distillation, nothing in sampling)
        uint32_t w[4] = {NONE, NONE, NONE, NONE};
        if (j + PER > 0 && j < n) {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (j + e >= 0 && j + e < n) {
                    if constexpr (sizeof(T) == 4)
                        w[e] = __float_as_uint(x[j + e]);
                    else
                        w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | (uint32_t)x[j + e] << 16 : (w[e / 2] & 0xFFFF0000u) | x[j + e];
                }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // f(logit, index) for every element of this lane's i-th piece, of all its pieces
    template <typename F>
    __device__ __forceinline__ void piece(int i, F f) const {
        float v[PER];
        unpack<T>(load(i), v);
        const int j = index(i);
#pragma unroll
        for (int e = 0; e < PER; ++e) f(v[e], j + e);
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        for (int i = 0; i < rounds; ++i) piece(i, f);
    }
    // f(logit, index) for the elements that are at least z_low, few of them
    template <typename F>
    __device__ __forceinline__ void each_from(float z_low, F f) const {
        for (int i = 0; i < rounds; ++i) from_piece<T>(load(i), index(i), z_low, f);
    }
};

// What stands on both sides is not mixed by the compiler: four logits at a time fill the pipelines, more of them take registers that spill.
__device__ __forceinline__ void apart() { __builtin_amdgcn_sched_barrier(0); }

// p or q, by value (a conditional assignment of the whole piece may become a choice between two addresses, and the pieces go to memory).
__device__ __forceinline__ uint4 choose(bool first, uint4 p, uint4 q) {
    const uint32_t m = 0u - (uint32_t)first;
    return make_uint4((p.x & m) | (q.x & ~m), (p.y & m) | (q.y & ~m), (p.z & m) | (q.z & ~m), (p.w & m) | (q.w & ~m));
}

// The same row, or part, in registers: at most N pieces a lane.
template <typename T, int N>
struct HeldRow : Row<T> {
    using Row<T>::PER;
    uint4 raw[N];

    __device__ __forceinline__ HeldRow(const LogitRows &in, long row, int wave, int waves, int lane, int from = 0, int most = 0x7FFFFFFF)
        : Row<T>(in, row, wave, waves, lane, from, most) {
        // whole pieces first, all in flight together; then the row's ends
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = this->index(i);
            raw[i] = make_uint4(Row<T>::NONE, Row<T>::NONE, Row<T>::NONE, Row<T>::NONE);
            if (i < this->rounds && j >= 0 && j + PER <= this->n) raw[i] = *reinterpret_cast<const uint4 *>(this->x + j);
        }
        if (this->first == 0 && this->lead > 0) raw[0] = this->load(0);
        const int i_end = partial_end();
        if (i_end >= 0) {
            const uint4 r = this->load(i_end);
#pragma unroll
            for (int i = 0; i < N; ++i) raw[i] = choose(i == i_end, r, raw[i]);
        }
    }
    // Round of this lane's piece that holds the row's last element, if it is partly outside the row; else -1.
    __device__ __forceinline__ int partial_end() const {
        const int d = (this->n + this->lead - 1) / PER - this->first;
        const int i = d >> 6;
        return (d & 63) == 0 && i >= 0 && i < this->rounds && this->index(i) + PER > this->n ? i : -1;
    }
    __device__ __forceinline__ void only_infinite() {
#pragma unroll
        for (int i = 0; i < N; ++i) raw[i] = share_infinite<T>(raw[i]);
    }
    __device__ __forceinline__ void none() {  // all -inf
#pragma unroll
        for (int i = 0; i < N; ++i) raw[i] = make_uint4(Row<T>::NONE, Row<T>::NONE, Row<T>::NONE, Row<T>::NONE);
    }
    template <typename F>
    __device__ __forceinline__ void each_piece(F f) const {  // f(logits, index of the first)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < this->rounds) {
                float v[PER];
                unpack<T>(raw[i], v);
                f(v, this->index(i));
                apart();
            }
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        each_piece([&](const float(&v)[PER], int j) {
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                f(v[e], j + e);
                if (e % 4 == 3) apart();
            }
        });
    }
    template <typename F>
    __device__ __forceinline__ void each_from(float z_low, F f) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < this->rounds) from_piece<T>(raw[i], this->index(i), z_low, f);
    }
};

// ------------------------------------------------------------------ sums over a wave and a workgroup (the same in every run)

// A value of 4 or 8 bytes from the lane that the pattern names; `other` where there is none or the row is masked out.
template <int PATTERN, int ROWS, typename V>
__device__ __forceinline__ V from_lane(V other, V v) {
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, other), __builtin_bit_cast(int, v), PATTERN, ROWS, 0xF, false));
    } else {
        const int2 o = __builtin_bit_cast(int2, other), a = __builtin_bit_cast(int2, v);
        int2 r;
        r.x = __builtin_amdgcn_update_dpp(o.x, a.x, PATTERN, ROWS, 0xF, false);
        r.y = __builtin_amdgcn_update_dpp(o.y, a.y, PATTERN, ROWS, 0xF, false);
        return __builtin_bit_cast(V, r);
    }
}
template <typename V>
__device__ __forceinline__ V read_lane(V v, int lane) {
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const int2 a = __builtin_bit_cast(int2, v);
        int2 r;
        r.x = __builtin_amdgcn_readlane(a.x, lane), r.y = __builtin_amdgcn_readlane(a.y, lane);
        return __builtin_bit_cast(V, r);
    }
}

// f over all lanes of the wave: within rows of 16 by exchanges, then over the four rows.
template <typename V, typename F>
__device__ __forceinline__ V wave_all(V v, F f) {
    v = f(v, from_lane<0xB1, 0xF>(v, v));   // neighbours
    v = f(v, from_lane<0x4E, 0xF>(v, v));   // pairs of four
    v = f(v, from_lane<0x141, 0xF>(v, v));  // mirrored halves of a row
    v = f(v, from_lane<0x140, 0xF>(v, v));  // mirrored rows
    return f(f(read_lane(v, 0), read_lane(v, 16)), f(read_lane(v, 32), read_lane(v, 48)));
}
template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
    return wave_all(v, [](V a, V b) { return a + b; });
}
// Sum over this lane and those before it.
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
    v += from_lane<0x111, 0xF>(V(0), v);  // the lane 1, 2, 4, 8 before, within the row
    v += from_lane<0x112, 0xF>(V(0), v);
    v += from_lane<0x114, 0xF>(V(0), v);
    v += from_lane<0x118, 0xF>(V(0), v);
    v += from_lane<0x142, 0xA>(V(0), v);  // last lane of the row before, to rows 1 and 3
    v += from_lane<0x143, 0xC>(V(0), v);  // lane 31, to rows 2 and 3
    return v;
}

// f over what the waves of a workgroup left in LDS: one read and exchanges within a row of lanes.
template <int WAVES, typename V, typename F>
__device__ __forceinline__ V over_lanes(V v, F f) {  // lanes w + i * WAVES hold the same value
    static_assert(WAVES == 1 || WAVES == 2 || WAVES == 4 || WAVES == 8 || WAVES == 16, "a row of lanes");
    if constexpr (WAVES >= 2) v = f(v, from_lane<0xB1, 0xF>(v, v));
    if constexpr (WAVES >= 4) v = f(v, from_lane<0x4E, 0xF>(v, v));
    if constexpr (WAVES >= 8) v = f(v, from_lane<0x141, 0xF>(v, v));
    if constexpr (WAVES >= 16) v = f(v, from_lane<0x140, 0xF>(v, v));
    return read_lane(v, 0);
}
template <int WAVES, typename V, typename F>
__device__ __forceinline__ V across_waves(const V *part, F f) {
    return over_lanes<WAVES>(part[threadIdx.x & (WAVES - 1)], f);
}
template <int WAVES, typename V>
__device__ __forceinline__ V sum_across(const V *part) {
    return across_waves<WAVES>(part, [](V a, V b) { return a + b; });
}
// Sum of what the waves before this one left.
template <int WAVES, typename V>
__device__ __forceinline__ V sum_before(const V *part) {
    const int w = threadIdx.x & (WAVES - 1);
    const V masked = w < (int)(threadIdx.x >> 6) ? part[w] : V(0);
    return over_lanes<WAVES>(masked, [](V a, V b) { return a + b; });
}

// f over all threads of the workgroup.  part: LDS, one entry per wave; free again after the next barrier.
template <int THREADS, typename V, typename F>
__device__ __forceinline__ V block_all(V v, V *part, F f) {
    v = wave_all(v, f);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return across_waves<THREADS / 64>(part, f);
}
template <int THREADS, typename V>
__device__ __forceinline__ V block_sum(V v, V *part) {
    return block_all<THREADS>(v, part, [](V a, V b) { return a + b; });
}

}  // namespace sushi
