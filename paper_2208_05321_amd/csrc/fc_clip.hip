// Global norm of a list of tensors, and clipping by it.
//
//   N = sqrt(sum over all elements of g^2),   g' = g * min(1, max_norm / (N + 1e-6))
//
// Squares are added up in 64 bits: sums of 1e9 elements keep their digits, and elements beyond 1.8e19, whose squares leave 32-bit
// floats, count.  Two passes, as the factor depends on every element: k_clip_norm leaves a sum per workgroup, k_clip_scale adds those up
// in every workgroup, in the same order, and scales.  Both are bound by HBM.
#include "dense_device.h"

#include <algorithm>
#include <math.h>

namespace fc {

constexpr int CLIP_THREADS = 256;
constexpr int CLIP_GROUP = 96;                     // tensors that one launch's arguments can describe (a launch takes 4 KB of them)
constexpr int CLIP_BLOCKS = 2048;                  // workgroups of the norm, for all launches of a call together

struct ClipTensor { const void* src; void* dst; int64_t size; int64_t begin; };      // begin: its first tile (see CLIP_TILE); type in the top bits of size
constexpr int64_t CLIP_TILE = 8192;                // elements; a tile belongs to one tensor
struct ClipGroup { ClipTensor t[CLIP_GROUP]; int count; int64_t tiles; };

__device__ __forceinline__ int clip_type(const ClipTensor& t) { return (int)(t.size >> 60); }
__device__ __forceinline__ int64_t clip_size(const ClipTensor& t) { return t.size & (((int64_t)1 << 60) - 1); }

// the tensor that tile k belongs to
__device__ __forceinline__ int clip_find(const ClipTensor* __restrict__ t, int count, int64_t tile) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t[mid].begin <= tile) lo = mid; else hi = mid;
    }
    return lo;
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

template <class T>
__device__ __forceinline__ double sum_squares(const T* __restrict__ p, int64_t n) {
    constexpr int N = VECTOR<T>;
    double s = 0;
    for (int64_t i = (int64_t)threadIdx.x * N; i < n; i += CLIP_THREADS * N) {
        float v[N];
        load_as_float(v, p + i, (int)min((int64_t)N, n - i));
#pragma unroll
        for (int k = 0; k < N; ++k) s = fma((double)v[k], (double)v[k], s);
    }
    return s;
}

// The first workgroup of the launch also leaves the tensors' descriptions in device memory, for k_clip_scale.
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_norm(ClipGroup g, ClipTensor* __restrict__ table, double* __restrict__ sums) {
    __shared__ double lds[CLIP_THREADS / 64];
    if (table && blockIdx.x == 0 && (int)threadIdx.x < g.count) table[threadIdx.x] = g.t[threadIdx.x];
    double s = 0;
    const int64_t base = g.t[0].begin;
    for (int64_t k = base + blockIdx.x; k < base + g.tiles; k += gridDim.x) {
        const ClipTensor& t = g.t[clip_find(g.t, g.count, k)];
        const int64_t at = (k - t.begin) * CLIP_TILE, n = min(CLIP_TILE, clip_size(t) - at);
        switch (clip_type(t)) {
            case FC_TYPE_F32: s += sum_squares((const float*)t.src + at, n); break;
            case FC_TYPE_BF16: s += sum_squares((const bf16*)t.src + at, n); break;
            default: s += sum_squares((const f16*)t.src + at, n); break;
        }
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

template <class T>
__device__ __forceinline__ void scale_tile(const T* src, T* dst, int64_t n, float factor) {
    constexpr int N = VECTOR<T>;
    for (int64_t i = (int64_t)threadIdx.x * N; i < n; i += CLIP_THREADS * N) {
        const int live = (int)min((int64_t)N, n - i);
        float v[N];
        load_as_float(v, src + i, live);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] *= factor;
        store_from_float(dst + i, v, live);
    }
}

__global__ __launch_bounds__(CLIP_THREADS) void k_clip_scale(const ClipTensor* __restrict__ table, int count, int64_t tiles, const double* __restrict__ sums,
                                                             int parts, float max_norm, float* __restrict__ norm_out) {
    __shared__ double lds[CLIP_THREADS / 64];
    double s = 0;
    for (int k = threadIdx.x; k < parts; k += CLIP_THREADS) s += sums[k];
    const double norm = sqrt(block_sum(s, lds));
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    if (isinf(max_norm) && !table) return;
    const double f = (double)max_norm / (norm + 1e-6);
    const float factor = isinf(max_norm) || f >= 1.0 ? 1.f : (float)f;        // (not a number stays one)
    for (int64_t k = blockIdx.x; k < tiles; k += gridDim.x) {
        const ClipTensor& t = table[clip_find(table, count, k)];
        if (factor == 1.f && t.src == t.dst) continue;
        const int64_t at = (k - t.begin) * CLIP_TILE, n = min(CLIP_TILE, clip_size(t) - at);
        switch (clip_type(t)) {
            case FC_TYPE_F32: scale_tile((const float*)t.src + at, (float*)t.dst + at, n, factor); break;
            case FC_TYPE_BF16: scale_tile((const bf16*)t.src + at, (bf16*)t.dst + at, n, factor); break;
            default: scale_tile((const f16*)t.src + at, (f16*)t.dst + at, n, factor); break;
        }
    }
}

static size_t clip_table_bytes(int64_t tensors) { return ((size_t)tensors * sizeof(ClipTensor) + 255) & ~(size_t)255; }
static int64_t clip_launches(int64_t tensors) { return cdiv(tensors, CLIP_GROUP); }
size_t clip_work_bytes(int64_t tensors) { return clip_table_bytes(tensors) + (size_t)(CLIP_BLOCKS + clip_launches(tensors) + 1) * sizeof(double); }

}  // namespace fc

using namespace fc;

extern "C" {

int grad_norm_clip(fc_dense* d, const void* const* grads_dev, void* const* out_dev, const int64_t* sizes, const int32_t* types, int32_t count,
                   float max_norm, float* norm_dev) {
    if (!d || count < 0 || !norm_dev || !(max_norm > 0.f) || (count > 0 && (!grads_dev || !sizes || !types))) return FC_ERR_INVALID_ARG;
    int64_t all_tiles = 0;
    for (int32_t k = 0; k < count; ++k) {
        if (sizes[k] < 0 || sizes[k] >= (int64_t)1 << 48 || !is_float_type(types[k]) || (sizes[k] > 0 && (!grads_dev[k] || (out_dev && !out_dev[k]))))
            return FC_ERR_INVALID_ARG;
        all_tiles += cdiv(sizes[k], CLIP_TILE);
    }
    FC_HIP(hipSetDevice(d->device));
    FC_TRY(dense_work(d, clip_work_bytes(count)));
    ClipTensor* table = reinterpret_cast<ClipTensor*>(d->work);
    double* sums = reinterpret_cast<double*>(d->work + clip_table_bytes(count));
    int64_t tile = 0, parts = 0, kept = 0;
    for (int32_t k = 0; k < count;) {
        ClipGroup g;
        g.count = 0; g.tiles = 0;
        for (; k < count && g.count < CLIP_GROUP; ++k) {
            if (sizes[k] == 0) continue;
            ClipTensor& t = g.t[g.count++];
            t.src = grads_dev[k]; t.dst = out_dev ? out_dev[k] : const_cast<void*>(grads_dev[k]);
            t.size = sizes[k] | (int64_t)types[k] << 60;
            t.begin = tile + g.tiles;
            g.tiles += cdiv(sizes[k], CLIP_TILE);
        }
        if (g.count == 0) continue;
        const int64_t blocks = std::max<int64_t>(1, std::min(g.tiles, CLIP_BLOCKS * g.tiles / all_tiles));
        k_clip_norm<<<(unsigned)blocks, CLIP_THREADS, 0, d->stream>>>(g, table + kept, sums + parts);
        tile += g.tiles; parts += blocks; kept += g.count;
    }
    const bool scales = tile > 0 && !(isinf(max_norm) && !out_dev);
    k_clip_scale<<<(unsigned)(scales ? std::min<int64_t>(tile, CLIP_BLOCKS) : 1), CLIP_THREADS, 0, d->stream>>>(scales ? table : nullptr, (int)kept, scales ? tile : 0, sums,
                                                                                                       (int)parts, max_norm, norm_dev);
    FC_HIP(hipGetLastError());
    return FC_OK;
}

}  // extern "C"
