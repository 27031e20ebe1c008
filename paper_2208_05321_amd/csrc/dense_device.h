// Shared by the operators beside the cached table (fc_token.hip, fc_norm.hip, fc_clip.hip): element types, vector accesses,
// sums over lanes, and the handle.
#pragma once

#include "fc_internal.h"

// Handle of the dense operators: a stream, the sticky flags, and device memory that calls use one after the other.
struct fc_dense {
    int device = 0;
    hipStream_t stream = nullptr;
    uint32_t* flags = nullptr;          // EF_ID_RANGE
    fc::SortBufs sort;                  // token_embed_bwd
    char* work = nullptr;               // what one call needs beyond that, laid out by the call
    size_t work_cap = 0;
    // A graph that was captured from calls of this handle holds addresses of its buffers: from the first capture on, buffers that are replaced by
    // larger ones are kept until the handle goes.
    bool captured = false;
    struct Kept { void* p; Kept* next; };
    Kept* kept = nullptr;
};

namespace fc {

using bf16 = __bf16;
using f16 = _Float16;

// N neighbouring elements, moved by one instruction wherever they start: rows may begin at any element (odd widths, odd strides, views), and
// the memory system takes 16 bytes at any address.  Against single elements for what is not aligned to 16 bytes this is one code path, and a row
// of 1111 16-bit columns moves as fast as one of 1112.
template <class T, int N> struct Pack { typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };

// columns that a lane takes at a time: 16 bytes of the source's type
template <class T> constexpr int VECTOR = 16 / (int)sizeof(T);

template <int N, class T>
__device__ __forceinline__ void load_vector(float (&v)[N], const T* __restrict__ p) {
    const auto x = *reinterpret_cast<const typename Pack<T, N>::V*>(p);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = (float)x[k];
}
template <int N, class T>
__device__ __forceinline__ void store_vector(T* __restrict__ p, const float (&v)[N]) {
    typename Pack<T, N>::V x;
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = (T)v[k];
    *reinterpret_cast<typename Pack<T, N>::V*>(p) = x;
}

// The same for the `live` first of N elements, one at least.  (The last one is read in the place of those beyond it, so that all loads are on their way
// together: in branches of their own each is waited for.)
template <int N, class T>
__device__ __forceinline__ void load_as_float(float (&v)[N], const T* __restrict__ p, int live) {
    if (live >= N) {
        const auto x = *reinterpret_cast<const typename Pack<T, N>::V*>(p);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (float)x[k];
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (float)p[k < live ? k : live - 1];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = k < live ? v[k] : 0.f;
    }
}
template <int N, class T>
__device__ __forceinline__ void store_from_float(T* __restrict__ p, const float (&v)[N], int live) {
    if (live >= N) {
        typename Pack<T, N>::V x;
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = (T)v[k];
        *reinterpret_cast<typename Pack<T, N>::V*>(p) = x;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) if (k < live) p[k] = (T)v[k];
    }
}

// Where a row's last two vectors overlap, a lane stores elements that another lane of the wavefront reads (in place, or added to): what was read
// before this is read before what is stored after it.  A wavefront's accesses leave in the order of its instructions; this keeps the compiler, which looks at one
// lane at a time, from changing that order, and is no instruction itself.
__device__ __forceinline__ void read_before_stores() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// f(), which the compiler does not merge with a like sequence of another branch: accesses that go past the caches and those that do not are one to it, and become ordinary ones.
template <int WHICH, class F>
__device__ __forceinline__ void apart(F f) {
    asm volatile("; %0" ::"i"(WHICH));
    f();
    asm volatile("; %0" ::"i"(WHICH));
}

// Sum over the wavefront's lanes, all of them active, in every lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ float add_lane(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float x) {
    x = add_lane<0x111, 0xf>(x);               // row_shr 1, 2, 4, 8
    x = add_lane<0x112, 0xf>(x);
    x = add_lane<0x114, 0xf>(x);
    x = add_lane<0x118, 0xf>(x);
    x = add_lane<0x142, 0xa>(x);               // row_bcast 15, 31
    x = add_lane<0x143, 0xc>(x);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
// Sum, or largest, over LANES neighbouring lanes (a power of two), in each of them.
template <int LANES> __device__ __forceinline__ float lanes_sum(float x) {
    if constexpr (LANES == 64) return wave_sum(x);
    else {
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) x += __shfl_xor(x, o);
        return x;
    }
}

inline int pow2_from(int64_t x, int most) { int p = 1; while (p < x && p < most) p <<= 1; return p; }

int dense_work(fc_dense* d, size_t bytes);     // d->work holds that many bytes
int dense_sort(fc_dense* d, int64_t n);        // d->sort holds n pairs
int dense_capturing(fc_dense* d, bool* now);   // whether the handle's stream is being captured
size_t token_work_bytes(int64_t n, int64_t rows, int64_t dim);
size_t norm_work_bytes(int64_t n, int64_t dim);
size_t clip_work_bytes(int64_t tensors);
size_t distill_work_bytes();                   // both whatever the sizes
size_t beam_work_bytes();

// Threads of one launch: the runtime takes fewer than 2^32.  Rows that need more go in several.
constexpr int64_t LAUNCH_THREADS = (int64_t)1 << 31;
constexpr int64_t DENSE_LIMIT = ((int64_t)1 << 31) - 65536;    // tokens, rows
constexpr int64_t DENSE_MAX_DIM = 1 << 20;

// One dispatch of a call's element types: f(T()) with T the type that `type` names.
template <class F>
int with_type(int32_t type, F f) {
    switch (type) {
        case FC_TYPE_F32: return f(float());
        case FC_TYPE_BF16: return f(bf16());
        case FC_TYPE_F16: return f(f16());
        default: return FC_ERR_INVALID_ARG;
    }
}
inline bool is_float_type(int32_t t) { return t == FC_TYPE_F32 || t == FC_TYPE_BF16 || t == FC_TYPE_F16; }
inline int type_bytes(int32_t t) { return t == FC_TYPE_F32 ? 4 : 2; }

}  // namespace fc
