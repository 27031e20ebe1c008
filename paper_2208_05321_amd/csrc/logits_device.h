// Shared by the operators on rows of logits (fc_distill.hip, fc_beam.hip): a slice of a row in registers, and sums of exponentials that are joined.
#pragma once

#include "dense_device.h"

#include <math.h>

namespace fc {

constexpr int LOGIT_THREADS = 256;                 // of a workgroup
constexpr float LOG2E = 1.44269504088896340736f;

__device__ __forceinline__ float wave_max(float x) {       // of numbers; in every lane
    auto step = [](float v, auto ctrl, auto rows) {
        const int o = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, -INFINITY), __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        return fmaxf(v, __builtin_bit_cast(float, o));
    };
    using std::integral_constant;
    x = step(x, integral_constant<int, 0x111>(), integral_constant<int, 0xf>());       // row_shr 1, 2, 4, 8
    x = step(x, integral_constant<int, 0x112>(), integral_constant<int, 0xf>());
    x = step(x, integral_constant<int, 0x114>(), integral_constant<int, 0xf>());
    x = step(x, integral_constant<int, 0x118>(), integral_constant<int, 0xf>());
    x = step(x, integral_constant<int, 0x142>(), integral_constant<int, 0xa>());       // row_bcast 15, 31
    x = step(x, integral_constant<int, 0x143>(), integral_constant<int, 0xc>());
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
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

    // stream: nobody reads the row again soon; it is kept out of the caches' way
    __device__ __forceinline__ void load(const T* row, int base, int lane, int dim, bool stream) {
        auto from = [&](int k) { return reinterpret_cast<const V*>(row + min(column(base, lane, k), dim - N)); };
        if (dim >= N && stream) {
#pragma unroll
            for (int k = 0; k < PER; ++k) x[k] = __builtin_nontemporal_load(from(k));
        } else if (dim >= N) {
#pragma unroll
            for (int k = 0; k < PER; ++k) x[k] = *from(k);
        } else {
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
    __device__ __forceinline__ float largest() const {
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) m = fmaxf(m, at(k, e));
        return m;
    }
    // sum of 2^(x c - off)
    __device__ __forceinline__ float exponentials(float c, float off) const {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) sum += __builtin_amdgcn_exp2f(fmaf(at(k, e), c, -off));
        return sum;
    }
    // Stores the slice, whose elements are results by now, but for the row's last vector where that is not a whole one; that is the business of one lane of the row, at the
    // end (code for it at every vector is most of a kernel).
    __device__ __forceinline__ void store(T* row, int base, int lane, int dim, bool stream) const {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int col = column(base, lane, k);
            if (col + N <= dim) {
                V* p = reinterpret_cast<V*>(row + col);
                if (stream) __builtin_nontemporal_store(x[k], p); else *p = x[k];
            }
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

}  // namespace fc
