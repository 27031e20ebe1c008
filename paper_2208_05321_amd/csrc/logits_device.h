// Shared by the operators on rows of logits (fc_distill.hip, fc_beam.hip): a slice of a row in registers, and sums of exponentials that are joined.
#pragma once

#include "dense_device.h"

#include <math.h>

namespace fc {

constexpr int LOGIT_THREADS = 256;                 // of a workgroup
constexpr float LOG2E = 1.44269504088896340736f;

// of numbers; in every lane.  (Lanes without a neighbour keep what they have.  Two wait states lie between a register's result and another lane's use of it.)
__device__ __forceinline__ float wave_max(float x) {
    asm("s_nop 1\n v_max_f32_dpp %0, %0, %0 row_shr:1 row_mask:0xf bank_mask:0xf\n"
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_shr:2 row_mask:0xf bank_mask:0xf\n"
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_shr:4 row_mask:0xf bank_mask:0xf\n"
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_shr:8 row_mask:0xf bank_mask:0xf\n"
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_bcast:15 row_mask:0xa bank_mask:0xf\n"
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_bcast:31 row_mask:0xc bank_mask:0xf\n"
        "s_nop 1" : "+v"(x));
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// A number (a lane's, for instance) as a value of this place of the program: what follows from it is worked out here, and not kept in registers from before a loop, or for after it.
template <class N>
__device__ __forceinline__ N here(N n) {
    asm volatile("" : "+v"(n));
    return n;
}

// A number that all of a wavefront's lanes have, in a scalar register.
__device__ __forceinline__ float scalar(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }

// The largest of three; NaN only if all are.  (Written as one instruction: of maxima of elements of 16 bits the compiler makes maxima in 16 bits, and of those, in bf16,
// maxima in 32 bits that are converted back each, three instructions more an element.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Waits of the LANES threads that share a row for one another: a wavefront's accesses leave in the order of its instructions, so that one
// only has to keep the compiler from changing that order.
template <int LANES>
__device__ __forceinline__ void row_sync() {
    if constexpr (LANES <= 64) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    else __syncthreads();
}

// PER vectors of 16 bytes for each of LANES lanes: one slice of a row.  All loads are on their way together.  Vectors lie LANES apart.  The row's
// last vector ends with the row (it overlaps the one before), those beyond it are loaded in its place; their first `skip` elements, which belong to
// others or are not there, become -infinity.  Rows that are shorter than a vector are read element by element.
template <class T, int LANES, int PER>
struct RowSlice {
    static constexpr int N = VECTOR<T>;
    static constexpr int COLUMNS = LANES * PER * N;
    typedef typename Pack<T, N>::V V;
    V x[PER];

    // the column that vector k of this lane begins at, and how many of its elements do not count (N: none does)
    static __device__ __forceinline__ int column(int base, int lane, int k) { return base + (k * LANES + lane) * N; }
    static __device__ __forceinline__ int skip(int col, int dim) { return min(max(col - (dim - N), 0), N); }

    // f(k, vector k's address) of a whole slice: the wavefront's lanes share an address but for 16 bytes times their number, which leaves 64-bit addresses out of the vector registers
    template <class P, class F>
    static __device__ __forceinline__ void each(P* row, int base, int lane, F f) {
        P* p = row + base;
#pragma unroll
        for (int k = 0; k < PER; ++k) f(k, p + k * LANES * N + (uint32_t)lane * N);
    }
    // of a row of a vector at least; stream: nobody reads the row again soon; it is kept out of the caches' way
    __device__ __forceinline__ void load_long(const T* row, int base, int lane, int dim, bool stream) {
        auto plain = [&](int k, const T* p) { x[k] = *reinterpret_cast<const V*>(p); };
        auto past = [&](int k, const T* p) { x[k] = __builtin_nontemporal_load(reinterpret_cast<const V*>(p)); };
        auto some = [&](auto get) {                // of a slice that the row ends in; what is beyond the row is not asked for
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int from = base + k * LANES * N;
                if (from < dim) get(k, row + min(column(base, lane, k), dim - N));
                else
#pragma unroll
                    for (int e = 0; e < N; ++e) x[k][e] = (T)-INFINITY;
            }
        };
        if (base + COLUMNS > dim) {
            if (stream) apart<2>([&] { some(past); });
            else apart<3>([&] { some(plain); });
        } else if (stream) apart<1>([&] { each(row, base, lane, past); });
        else apart<0>([&] { each(row, base, lane, plain); });
    }
    __device__ __forceinline__ void load(const T* row, int base, int lane, int dim, bool stream) {
        if (dim >= N) load_long(row, base, lane, dim, stream);
        else {
#pragma unroll
            for (int k = 0; k < PER; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) x[k][e] = row[max(dim - N + e, 0)];
        }
    }
    __device__ __forceinline__ void cut(int base, int lane, int dim) {
        if (base + COLUMNS <= dim) return;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (dim >= N && (base + (k + 1) * LANES * N <= dim || base + k * LANES * N >= dim)) continue;       // (all of the lanes' vectors are whole, or none is there)
            const int s = skip(column(base, lane, k), dim);
#pragma unroll
            for (int e = 0; e < N; ++e) if (e < s) x[k][e] = (T)-INFINITY;
        }
    }
    __device__ __forceinline__ float at(int k, int e) const { return (float)x[k][e]; }
    // Between two passes over the registers: what the one has converted to 32 bits is not kept for the other, which converts again.  (Kept, 64 elements of 16 bits take 64
    // registers more, and a row of 1024 threads does not fit in them.)
    __device__ __forceinline__ void forget() {
        typedef uint32_t W __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            W w = __builtin_bit_cast(W, x[k]);
            asm volatile("" : "+v"(w));
            x[k] = __builtin_bit_cast(V, w);
        }
    }
    // one of the vectors, by a number that is not known beforehand
    __device__ __forceinline__ V pick(int k) const {
        V v = x[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) {
            const V y = x[j];                      // (read before it is asked for: else the compiler makes the registers memory, to read the one)
            v = j == k ? y : v;
        }
        return v;
    }
    __device__ __forceinline__ float largest(int k) const {
        float m = -INFINITY;
#pragma unroll
        for (int e = 0; e < N; e += 2) m = max3(m, at(k, e), at(k, e + 1));
        return m;
    }
    // The largest element.  (Elements of 16 bits are compared as integers, two at a time, without being converted.  In that order the numbers of sign 0 come as they are, above
    // those of sign 1, which come the other way round: where all are of sign 1 the largest is the smallest of their bits.)
    typedef int16_t I2 __attribute__((ext_vector_type(2)));
    typedef uint16_t U2 __attribute__((ext_vector_type(2)));
    template <class F>
    __device__ __forceinline__ void pairs(int k, F f) const {
        typedef uint32_t W __attribute__((ext_vector_type(4)));
        const W w = __builtin_bit_cast(W, x[k]);
        const uint32_t p[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) f(p[j]);
    }
    __device__ __forceinline__ I2 largest_pair(int k) const {
        I2 i = I2{INT16_MIN, INT16_MIN};
        pairs(k, [&](uint32_t p) { i = __builtin_elementwise_max(i, __builtin_bit_cast(I2, p)); });
        return i;
    }
    __device__ __forceinline__ float largest() const {
        if constexpr (sizeof(T) == 2) {
            I2 i = largest_pair(0);
#pragma unroll
            for (int k = 1; k < PER; ++k) i = __builtin_elementwise_max(i, largest_pair(k));
            int16_t best = i[0] > i[1] ? i[0] : i[1];
            if (best < 0) {
                U2 u = U2{UINT16_MAX, UINT16_MAX};
#pragma unroll
                for (int k = 0; k < PER; ++k) pairs(k, [&](uint32_t p) { u = __builtin_elementwise_min(u, __builtin_bit_cast(U2, p)); });
                best = (int16_t)(u[0] < u[1] ? u[0] : u[1]);
            }
            return (float)__builtin_bit_cast(T, best);
        } else {
            float m = -INFINITY;
#pragma unroll
            for (int k = 0; k < PER; k += 2) m = max3(m, largest(k), largest(k + 1));
            return m;
        }
    }
    // A bit for each vector that has an element of `least` or more.
    __device__ __forceinline__ uint32_t vectors_from(float least) const {
        uint32_t at = 0;
        if constexpr (sizeof(T) == 2)
            if (least > 0.f) {                     // (all of sign 0, then: integers again)
                const T t = (T)least;
                const int16_t below = (int16_t)(__builtin_bit_cast(int16_t, t) - ((float)t >= least ? 1 : 0));
                const I2 b = I2{below, below};
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (__builtin_bit_cast(uint32_t, __builtin_elementwise_max(largest_pair(k), b)) != __builtin_bit_cast(uint32_t, b)) at |= 1u << k;
                return at;
            }
#pragma unroll
        for (int k = 0; k < PER; ++k) if (largest(k) >= least) at |= 1u << k;
        return at;
    }
    // sum of 2^(x c - off); 64 elements are added one after the other, at most
    __device__ __forceinline__ float exponentials(float c, float off) const {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < PER; j += 64 / N) {
            float part = 0.f;
#pragma unroll
            for (int k = j; k < j + 64 / N && k < PER; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) part += __builtin_amdgcn_exp2f(fmaf(at(k, e), c, -off));
            sum = j ? sum + part : part;
        }
        return sum;
    }
    // Stores the slice, whose elements are results by now, but for the row's last vector where that is not a whole one; that is the business of one lane of the row, at the
    // end (code for it at every vector is most of a kernel).
    __device__ __forceinline__ void store(T* row, int base, int lane, int dim, bool stream) const {
        auto plain = [&](int k, T* p) { *reinterpret_cast<V*>(p) = x[k]; };
        auto past = [&](int k, T* p) { __builtin_nontemporal_store(x[k], reinterpret_cast<V*>(p)); };
        if (base + COLUMNS <= dim) {
            if (stream) apart<1>([&] { each(row, base, lane, past); });
            else apart<0>([&] { each(row, base, lane, plain); });
            return;
        }
        lane = here(lane);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int col = column(base, lane, k);
            if (col + N <= dim) plain(k, row + col);
        }
        const int whole = dim - dim % N, last = (whole - base) / N;
        if (whole < dim && whole >= base && whole < base + COLUMNS && last % LANES == lane) {
            const V v = pick(last / LANES);        // ends with the row
#pragma unroll
            for (int e = 0; e < N; ++e) if (dim - N + e >= whole) row[dim - N + e] = v[e];
        }
    }
};

// exponentials are taken from `from`: the largest element, or 0 where all are -infinity
__device__ __forceinline__ float from_of(float m) { return m == -INFINITY ? 0.f : m; }

// How exponentials are taken from an element `from`, the largest: 2^(c (x - from)) = back * 2^(fma(x, scale, -off)), one instruction before an element's exponential, where a difference first and
// its product would be two.  off is the rounded product of `from`, and back mends its rounding, which reaches 2^32 where the product reaches 2^30, and beyond the range of numbers further out.  From there on elements
// are so far apart (2^-24 of themselves at least: 64 and more in the exponent) that only those equal to the largest count: scale is a power of two then, which makes the products exact, and they are some
// 2^40, which leaves nothing of the others.  (c: log2(e) over a temperature of 1/1024 to 1024.)  Infinite or no number: all exponentials are none.
struct Exponents { float scale, off, back; };
__device__ __forceinline__ Exponents exponents(float from, float c) {
    from = from_of(from);
    const float off = from * c;
    const bool far = !(fabsf(off) < 0x1p30f);
    const float scale = far ? __builtin_bit_cast(float, (294u << 23) - (__builtin_bit_cast(uint32_t, from) & 0x7f800000u)) : c;      // 2^(40 - from's exponent)
    const float o = far ? from * scale : off;
    return Exponents{scale, o, __builtin_amdgcn_exp2f(fmaf(-from, scale, o))};
}
// What a sum of exponentials from `from` counts as in one from `to`, no smaller.
__device__ __forceinline__ float part_of(float from, float to, float c) { return __builtin_amdgcn_exp2f((from - from_of(to)) * c); }

}  // namespace fc
