// Global norm of a list of tensors, and clipping by it.
//
//   N = sqrt(sum over all elements of g^2),   g' = g * min(1, max_norm / (N + 1e-6))
//
// Squares are added up in 64 bits: sums of 1e9 elements keep their digits, and elements beyond 1.8e19, whose squares leave 32-bit
// floats, count.  Two passes, as the factor depends on every element: k_clip_norm leaves a sum per workgroup, k_clip_scale adds those up
// in every workgroup, in the same order, and scales.  Both are bound by HBM: 906 MB of bf16 and f32 in 240 tensors, norm 188 us (4.8 TB/s), scale 338 us
// (5.4 TB/s).  Few elements: the two launches, 5 and 7 us at 8 MB.
#include "dense_device.h"

#include <algorithm>
#include <math.h>

#include <type_traits>

namespace fc {

constexpr int CLIP_THREADS = 256;
constexpr int CLIP_GROUP = 120;                    // tensors that one launch's arguments can describe (a launch takes 4 KB of them)
// us a call.  Workgroups, 1024 / 2048 / 4096 at most: 20 f32 tensors of 1 M elements 42.5 / 46.8 / 46.0, 240 of 1.9 M bf16 548 / 549 / 541, 20 of 105 k f32 13.9 / 13.7 / 13.8.
// Elements of a tile, 4096 / 8192 / 16,384: 45.0 / 46.8 / 42.5, 562 / 549 / 546, 12.0 / 13.7 / 13.5, one of 4 M bf16 10.4 / 9.2 / 9.2.
constexpr int CLIP_BLOCKS = 2048;                  // workgroups
constexpr int64_t CLIP_TILE = 8192;                // elements; a tile belongs to one tensor

struct ClipTensor { const void* src; void* dst; int64_t size, begin; };      // size: elements, the type in the top bits; begin: its first tile
struct ClipGroup { ClipTensor t[CLIP_GROUP]; int count; };
static_assert(sizeof(ClipGroup) + 64 <= 4096, "arguments of a launch");

__device__ __forceinline__ int clip_type(const ClipTensor& t) { return (int)(t.size >> 60); }
__device__ __forceinline__ int64_t clip_size(const ClipTensor& t) { return t.size & (((int64_t)1 << 60) - 1); }

// f(tensor, first element of the tile, elements) for a workgroup's share of the tiles, which are neighbours: the tensor of the first is looked
// up, the others follow.  Looked up for each, in turn with the other workgroups', every 16 KB waited for a chain of eight loads.
template <class F>
__device__ __forceinline__ void clip_tiles(const ClipTensor* __restrict__ t, int count, int64_t tiles, unsigned share, F f) {
    const int64_t k0 = tiles * share / gridDim.x, k1 = tiles * (share + 1) / gridDim.x;
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t[mid].begin <= k0) lo = mid; else hi = mid;
    }
    for (int64_t k = k0; k < k1; ++k) {
        while (lo + 1 < count && t[lo + 1].begin <= k) ++lo;
        const int64_t at = (k - t[lo].begin) * CLIP_TILE;
        f(t[lo], at, min(CLIP_TILE, clip_size(t[lo]) - at));
    }
}

__device__ __forceinline__ double block_sum(double x, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int k = 0; k < CLIP_THREADS / 64; ++k) s += lds[k];
    __syncthreads();
    return s;
}

// f(vector) for each of a lane's vectors of p[0 .. n); those of a whole tile are all on their way together
template <class T, class F>
__device__ __forceinline__ void clip_vectors(const T* __restrict__ p, int64_t n, F f) {
    constexpr int N = VECTOR<T>, STEP = CLIP_THREADS * N, PER = (int)(CLIP_TILE / STEP);
    if (n == CLIP_TILE) {
        typename Pack<T, N>::V x[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) x[k] = *reinterpret_cast<const typename Pack<T, N>::V*>(p + k * STEP + threadIdx.x * N);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = (float)x[k][e];
            f(v, k * STEP + (int)threadIdx.x * N, N);
        }
        return;
    }
    for (int i = threadIdx.x * N; i < n; i += STEP) {
        float v[N];
        load_as_float(v, p + i, (int)min((int64_t)N, n - i));
        f(v, i, (int)min((int64_t)N, n - i));
    }
}

template <class T>
__device__ __forceinline__ double sum_squares(const T* __restrict__ p, int64_t n) {
    constexpr int N = VECTOR<T>;
    double s = 0;
    clip_vectors(p, n, [&](const float (&v)[N], int, int) {
#pragma unroll
        for (int k = 0; k < N; ++k) s = fma((double)v[k], (double)v[k], s);
    });
    return s;
}

__device__ __forceinline__ double norm_tiles(const ClipTensor* __restrict__ t, int count, int64_t tiles) {
    double s = 0;
    clip_tiles(t, count, tiles, blockIdx.x, [&](const ClipTensor& q, int64_t at, int64_t n) {
        switch (clip_type(q)) {
            case FC_TYPE_F32: s += sum_squares((const float*)q.src + at, n); break;
            case FC_TYPE_BF16: s += sum_squares((const bf16*)q.src + at, n); break;
            default: s += sum_squares((const f16*)q.src + at, n); break;
        }
    });
    return s;
}

// Descriptions on their way to device memory, as arguments.
__global__ __launch_bounds__(128) void k_clip_table(ClipGroup g, ClipTensor* __restrict__ table) {
    if ((int)threadIdx.x < g.count) table[threadIdx.x] = g.t[threadIdx.x];
}

// ARGS: the tensors are those of the arguments, and the first workgroup leaves them in `table`; else the table holds them.
template <bool ARGS>
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_norm(std::conditional_t<ARGS, ClipGroup, int> g, ClipTensor* __restrict__ table, int64_t tiles, double* __restrict__ sums) {
    __shared__ double lds[CLIP_THREADS / 64];
    double s;
    if constexpr (ARGS) {
        if (blockIdx.x == 0 && (int)threadIdx.x < g.count) table[threadIdx.x] = g.t[threadIdx.x];
        s = norm_tiles(g.t, g.count, tiles);
    } else s = norm_tiles(table, g, tiles);
    s = block_sum(s, lds);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

template <class T>
__device__ __forceinline__ void scale_tile(const T* src, T* dst, int64_t n, float factor) {
    constexpr int N = VECTOR<T>;
    clip_vectors(src, n, [&](float (&v)[N], int at, int live) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] *= factor;
        store_from_float(dst + at, v, live);
    });
}

// (The last tiles first: they are what the memory-side cache holds of the pass before.)
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_scale(const ClipTensor* __restrict__ table, int count, int64_t tiles, const double* __restrict__ sums,
                                                             int parts, float max_norm, float* __restrict__ norm_out) {
    __shared__ double lds[CLIP_THREADS / 64];
    double s = 0;
    for (int k = threadIdx.x; k < parts; k += CLIP_THREADS) s += sums[k];
    const double norm = sqrt(block_sum(s, lds));
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const double f = (double)max_norm / (norm + 1e-6);
    const float factor = isinf(max_norm) || f >= 1.0 ? 1.f : (float)f;        // (not a number stays one)
    if (!table) return;
    clip_tiles(table, count, tiles, gridDim.x - 1 - blockIdx.x, [&](const ClipTensor& q, int64_t at, int64_t n) {
        if (factor == 1.f && q.src == q.dst) return;
        switch (clip_type(q)) {
            case FC_TYPE_F32: scale_tile((const float*)q.src + at, (float*)q.dst + at, n, factor); break;
            case FC_TYPE_BF16: scale_tile((const bf16*)q.src + at, (bf16*)q.dst + at, n, factor); break;
            default: scale_tile((const f16*)q.src + at, (f16*)q.dst + at, n, factor); break;
        }
    });
}

static size_t clip_table_bytes(int64_t tensors) { return ((size_t)tensors * sizeof(ClipTensor) + 255) & ~(size_t)255; }
size_t clip_work_bytes(int64_t tensors) { return clip_table_bytes(tensors) + CLIP_BLOCKS * sizeof(double); }

}  // namespace fc

using namespace fc;

extern "C" {

int grad_norm_clip(fc_dense* d, const void* const* grads_dev, void* const* out_dev, const int64_t* sizes, const int32_t* types, int32_t count,
                   float max_norm, float* norm_dev) {
    if (!d || count < 0 || !norm_dev || !(max_norm > 0.f) || (count > 0 && (!grads_dev || !sizes || !types))) return FC_ERR_INVALID_ARG;
    for (int32_t k = 0; k < count; ++k)
        if (sizes[k] < 0 || sizes[k] >= (int64_t)1 << 48 || !is_float_type(types[k]) || (sizes[k] > 0 && (!grads_dev[k] || (out_dev && !out_dev[k]))))
            return FC_ERR_INVALID_ARG;
    FC_HIP(hipSetDevice(d->device));
    FC_TRY(dense_work(d, clip_work_bytes(count)));
    const hipStream_t st = d->stream;
    ClipTensor* table = reinterpret_cast<ClipTensor*>(d->work);
    double* sums = reinterpret_cast<double*>(d->work + clip_table_bytes(count));
    int64_t tiles = 0;
    int kept = 0;
    ClipGroup g;
    g.count = 0;
    for (int32_t k = 0; k < count; ++k) {
        if (sizes[k] == 0) continue;
        if (g.count == CLIP_GROUP) {
            k_clip_table<<<1, 128, 0, st>>>(g, table + kept);
            kept += g.count;
            g.count = 0;
        }
        g.t[g.count++] = ClipTensor{grads_dev[k], out_dev ? out_dev[k] : const_cast<void*>(grads_dev[k]), sizes[k] | (int64_t)types[k] << 60, tiles};
        tiles += cdiv(sizes[k], CLIP_TILE);
    }
    const int parts = (int)std::min<int64_t>(tiles, CLIP_BLOCKS), total = kept + g.count;
    if (kept) {
        k_clip_table<<<1, 128, 0, st>>>(g, table + kept);
        k_clip_norm<false><<<parts, CLIP_THREADS, 0, st>>>(total, table, tiles, sums);
    } else if (parts) k_clip_norm<true><<<parts, CLIP_THREADS, 0, st>>>(g, table, tiles, sums);
    const bool scales = tiles > 0 && !(isinf(max_norm) && !out_dev);
    k_clip_scale<<<scales ? parts : 1, CLIP_THREADS, 0, st>>>(scales ? table : nullptr, total, tiles, sums, parts, max_norm, norm_dev);
    FC_HIP(hipGetLastError());
    return FC_OK;
}

}  // extern "C"
