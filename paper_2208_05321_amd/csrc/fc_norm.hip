// Root-mean-square norm with the residual's addition, results in 8 bits with scales, and the backward pass.
//
//   forward   h = T(x + r),  rho = (mean(h^2) + eps)^-1/2,  y = h * rho * w
//             8 bits: s = max |y| / qmax over the row or over each group of columns, q = Q(y / s)
//   backward  c = dy * w,  dh = dh_in + rho * (c - h * rho^2 * mean(c * h)),  dw = sum over the rows of dy * h * rho
//
// A row stays in registers between the sums and the results, so each input is read once and each result written once: HBM bounds a
// large call, the launch a small one.  Lanes of a row: as many as there are vectors of 16 bytes, up to a wavefront; wider rows take
// a workgroup.  The norm is that of the stored h, so that the backward pass, which works rho out again, sees what the forward pass saw.
#include "dense_device.h"

#include <algorithm>
#include <float.h>
#include <math.h>

#include <type_traits>

namespace fc {

struct F8 { uint8_t b; };                          // FC_TYPE_F8E4M3
template <class Q> constexpr float QMAX = 0.f;
template <> constexpr float QMAX<F8> = 448.f;
template <> constexpr float QMAX<int8_t> = 127.f;

// the larger one, or not a number if either is none
__device__ __forceinline__ float nan_max(float a, float b) { return a > b || a != a ? a : b; }

// threads of a workgroup: 256, or the TPR lanes of one row
constexpr int norm_threads(int tpr) { return tpr < 256 ? 256 : tpr; }

// What a row's last vector is.  WHOLE: the width is a multiple of N.  OVER: the vector ends with the row and overlaps the one before; its lane leaves the
// first `skip` elements out of every sum, and stores for them what the lane before stores.  That needs all of a row to be read before any of
// it is written (results may take the place of inputs), and rows of a vector at least; otherwise PART: the vector is loaded and stored element by
// element, in code that is four fifths of a kernel that has it (9 KB of instructions for 4096 16-bit columns, fetched once a launch: 4.1 us for a
// single row, 3.1 without) and takes registers: backward pass, 7227 rows of 2249 columns 65 us, of 2248 29; 31 this way.
enum NormEnd { WHOLE, OVER, PART };
template <int END, int N, class T>
__device__ __forceinline__ void load_some(float (&v)[N], const T* __restrict__ p, int live) {
    if constexpr (END != PART) load_vector(v, p);
    else load_as_float(v, p, live);
}
template <int END, int N, class T>
__device__ __forceinline__ void store_some(T* __restrict__ p, const float (&v)[N], int live) {
    if constexpr (END != PART) store_vector(p, v);
    else store_from_float(p, v, live);
}
// The vector that begins at column `v`: is it there, where does it begin, how many of its elements belong to the one before.
struct NormVector { bool in; int col, skip; };
template <int END, int N>
__device__ __forceinline__ NormVector norm_vector(int v, int dim) {
    if constexpr (END == OVER) { const int col = min(v, dim - N); return NormVector{v < dim, col, v - col}; }
    else return NormVector{v < dim, v, 0};
}
template <int END> __device__ __forceinline__ bool counts(const NormVector& q, int e) { return END != OVER || e >= q.skip; }

// Sum of x over the TPR lanes of a row, in each of them.  lds: TPR / 64 words for each of the two turns that alternate, so that one barrier a
// sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float* lds) {
    if constexpr (TPR <= 64) return lanes_sum<TPR>(x);
    else {
        x = wave_sum(x);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < TPR / 64; ++k) s += lds[k];
        return s;
    }
}
template <int TPR>
__device__ __forceinline__ void row_sums(float& x, float& y, float (*lds)[TPR > 64 ? TPR / 64 : 1]) {
    if constexpr (TPR <= 64) { x = lanes_sum<TPR>(x); y = lanes_sum<TPR>(y); }
    else {
        x = wave_sum(x); y = wave_sum(y);
        if ((threadIdx.x & 63) == 0) { lds[0][threadIdx.x >> 6] = x; lds[1][threadIdx.x >> 6] = y; }
        __syncthreads();
        x = y = 0.f;
#pragma unroll
        for (int k = 0; k < TPR / 64; ++k) { x += lds[0][k]; y += lds[1][k]; }
    }
}
template <int TPR>
__device__ __forceinline__ float row_max(float x, float* lds) {
#pragma unroll
    for (int o = 1; o < (TPR < 64 ? TPR : 64); o <<= 1) x = nan_max(x, __shfl_xor(x, o));
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = lds[0];
#pragma unroll
        for (int k = 1; k < TPR / 64; ++k) x = nan_max(x, lds[k]);
    }
    return x;
}

template <int END, class T, int N>
__device__ __forceinline__ void load_weight(float (&v)[N], const void* w, bool f32, int col, int live) {
    if (f32) load_some<END>(v, (const float*)w + col, live);
    else load_some<END>(v, (const T*)w + col, live);
}

// v / scale, rounded as a division is, in three instructions an element: the product with the rounded reciprocal, and what that leaves over, which is
// exact (scales from 1e-28 on), times the reciprocal again (Markstein's correction).  The product alone is off by up to 1.5 units of 32 bits, and a quotient that close to the
// middle between two 8-bit values then goes to the wrong one.  inv, by: 0 for a scale that is too small for a reciprocal or infinite.
// Quotients are at most QMAX and one unit of 32 bits (|v| <= m and scale = m / QMAX, rounded), which rounds to QMAX: nothing is cut off.
struct Quotient {
    float inv, by;
    __device__ __forceinline__ explicit Quotient(float scale) {
        inv = scale >= FLT_MIN || scale != scale ? 1.f / scale : 0.f;
        by = inv > 0.f ? scale : 0.f;
    }
    __device__ __forceinline__ float operator()(float v) const {
        const float t = v * inv;
        return fmaf(-fmaf(t, by, -v), inv, t);
    }
};

// (elements skip .. live - 1)
template <bool ALL, int N>
__device__ __forceinline__ void store_quantised(F8* p, const float (&v)[N], const Quotient& of, int skip, int live) {
    uint32_t word[N / 4];
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(of(v[k]), of(v[k + 1]), 0, false);
        word[k / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(of(v[k + 2]), of(v[k + 3]), x, true);
    }
    if (ALL || (skip == 0 && live >= N)) {
        typedef uint32_t V __attribute__((ext_vector_type(N / 4), aligned(1)));
        V x;
#pragma unroll
        for (int k = 0; k < N / 4; ++k) x[k] = word[k];
        *reinterpret_cast<V*>(p) = x;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) if (k >= skip && k < live) p[k].b = (uint8_t)(word[k / 4] >> (k % 4 * 8));
    }
}
template <bool ALL, int N>
__device__ __forceinline__ void store_quantised(int8_t* p, const float (&v)[N], const Quotient& of, int skip, int live) {
    typedef int8_t V __attribute__((ext_vector_type(N), aligned(1)));
    V x;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float t = rintf(of(v[k]));
        x[k] = (int8_t)(int)(t == t ? t : 0.f);
    }
    if (ALL || (skip == 0 && live >= N)) *reinterpret_cast<V*>(p) = x;
    else {
#pragma unroll
        for (int k = 0; k < N; ++k) if (k >= skip && k < live) p[k] = x[k];
    }
}

struct NormFwd {
    const void *x, *residual, *weight;
    void *h, *y;
    float* scales;
    int64_t x_stride, residual_stride, h_stride, y_stride, first, n;      // rows first .. n - 1
    int dim, weight_f32, group;          // group: columns of a scale, 0 = the row
    float eps;
};

// 8192 rows of 8192 bf16 columns with residual, to 8 bits by groups of 128: 97 to 99 us (472 MB, 4.8 TB/s); one row of 4096 3.2 us; 777 of 1111 f16 3.
// KEEP: vectors of a row that a lane keeps in registers, 0: rows too wide for that, h is worked out again for each of the steps (with END PART)
template <int TPR, int KEEP, int END, class T, class Q>
__global__ __launch_bounds__(norm_threads(TPR)) void k_norm_fwd(NormFwd a) {
    constexpr int N = VECTOR<T>, NT = norm_threads(TPR), K = KEEP ? KEEP : 1;
    constexpr bool QUANT = QMAX<Q> > 0.f;
    static_assert(KEEP > 0 || END == PART, "lanes that share columns read them before they write");
    __shared__ float lds[2][TPR > 64 ? TPR / 64 : 1];
    const int lane = threadIdx.x & (TPR - 1);
    const int64_t row = a.first + (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
    if (TPR <= 64 && row >= a.n) return;          // (whole rows of lanes; a workgroup with one row always has it)
    const T* const x = (const T*)a.x + row * a.x_stride;
    const T* const r = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
    T* const h = a.h ? (T*)a.h + row * a.h_stride : nullptr;
    Q* const y = (Q*)a.y + row * a.y_stride;
    const int vectors = KEEP ? KEEP : (a.dim + TPR * N - 1) / (TPR * N);
    float v[K][N];
    auto vector = [&](int k) { return norm_vector<END, N>((k * TPR + lane) * N, a.dim); };
    auto fetch = [&](float (&t)[N], int col) {
        const int live = a.dim - col;
        load_some<END>(t, x + col, live);
        if (r) {
            float s[N];
            load_some<END>(s, r + col, live);
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = (float)(T)(t[e] + s[e]);
        }
    };
    float s = 0.f;
#pragma unroll K
    for (int k = 0; k < (KEEP ? KEEP : vectors); ++k) {
        const NormVector q = vector(k);
        float (&t)[N] = v[KEEP ? k : 0];
        if (q.in) fetch(t, q.col);
        else
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) s = counts<END>(q, e) ? fmaf(t[e], t[e], s) : s;
    }
    const float rho = rsqrtf(row_sum<TPR>(s, lds[0]) / (float)a.dim + a.eps);
    auto result = [&](float (&t)[N], int col) {                      // h -> y
        float w[N];
        load_weight<END, T>(w, a.weight, a.weight_f32, col, a.dim - col);
#pragma unroll
        for (int e = 0; e < N; ++e) t[e] = t[e] * rho * w[e];
    };
    auto store_h = [&](int col) {                                    // KEEP 0: h once more, when it is read no more
        if (KEEP || !h) return;
        float t[N];
        fetch(t, col);
        store_some<END>(h + col, t, a.dim - col);
    };
    float most = 0.f;
#pragma unroll K
    for (int k = 0; k < (KEEP ? KEEP : vectors); ++k) {
        const NormVector q = vector(k);
        float (&t)[N] = v[KEEP ? k : 0];
        if (q.in) {
            if (!KEEP) fetch(t, q.col);
            if (KEEP && h) store_some<END>(h + q.col, t, a.dim - q.col);
            result(t, q.col);
            if constexpr (!QUANT) {
                store_h(q.col);
                store_some<END>(y + q.col, t, a.dim - q.col);
            } else
#pragma unroll
                for (int e = 0; e < N; ++e) most = counts<END>(q, e) ? nan_max(fabsf(t[e]), most) : most;
        }
        if constexpr (QUANT) {
            if (a.group) {                                           // neighbouring lanes hold a group's columns
                float m = most;
                const int lanes = min(a.group / N, TPR < 64 ? TPR : 64);
                for (int o = 1; o < lanes; o <<= 1) m = nan_max(m, __shfl_xor(m, o));
                most = 0.f;
                if (q.in) {
                    const float scale = m / QMAX<Q>;
                    const int at = q.col + q.skip;
                    if (at % a.group == 0) a.scales[row * ((a.dim + a.group - 1) / a.group) + at / a.group] = scale;
                    store_h(q.col);
                    store_quantised<END == WHOLE>(y + q.col, t, Quotient(scale), q.skip, a.dim - q.col);
                }
            }
        }
    }
    if constexpr (QUANT) {
        if (a.group) return;
        const float scale = row_max<TPR>(most, lds[1]) / QMAX<Q>;
        const Quotient of(scale);
        if (lane == 0) a.scales[row] = scale;
#pragma unroll K
        for (int k = 0; k < (KEEP ? KEEP : vectors); ++k) {
            const NormVector q = vector(k);
            float (&t)[N] = v[KEEP ? k : 0];
            if (!q.in) continue;
            if (!KEEP) { fetch(t, q.col); result(t, q.col); }
            store_h(q.col);
            store_quantised<END != PART>(y + q.col, t, of, 0, a.dim - q.col);
        }
    }
}

struct NormBwd {
    const void *dy, *h, *weight, *dh_in;
    void* dx;
    float* part;                         // [workgroups][dim]
    int64_t dy_stride, h_stride, dh_in_stride, dx_stride, n;
    int dim, weight_f32;
    float eps;
};

// The weight's gradient is summed over the workgroup's rows in registers and then over the workgroups by k_norm_dw: no atomics, the same order always.
// 16,384 rows of 4096 bf16 columns 97 to 100 us (537 MB, 5.4 TB/s), and 6 for k_norm_dw.
// KEEP as above; with 0 a workgroup adds to its row of `part` in memory
template <int TPR, int KEEP, int END, class T>
__global__ __launch_bounds__(norm_threads(TPR)) void k_norm_bwd(NormBwd a) {
    constexpr int N = VECTOR<T>, NT = norm_threads(TPR), GROUPS = NT / TPR, K = KEEP ? KEEP : 1;
    static_assert(KEEP > 0 || END == PART, "lanes that share columns read them before they write");
    __shared__ float lds[4][TPR > 64 ? TPR / 64 : 1];
    __shared__ float cols[GROUPS > 1 ? GROUPS * TPR * K * N : 1];
    const int lane = threadIdx.x & (TPR - 1);
    const int vectors = KEEP ? KEEP : (a.dim + TPR * N - 1) / (TPR * N);
    float* const part = a.part + (size_t)blockIdx.x * a.dim;
    auto vector = [&](int k) { return norm_vector<END, N>((k * TPR + lane) * N, a.dim); };
    float w[K][N], dw[K][N];
    if (KEEP) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const NormVector q = vector(k);
            if (q.in) load_weight<END, T>(w[k], a.weight, a.weight_f32, q.col, a.dim - q.col);
#pragma unroll
            for (int e = 0; e < N; ++e) { if (!q.in) w[k][e] = 0.f; dw[k][e] = 0.f; }
        }
    } else
        for (int col = threadIdx.x; col < a.dim; col += NT) part[col] = 0.f;
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * GROUPS; row0 < a.n; row0 += (int64_t)gridDim.x * GROUPS, turn ^= 2) {
        const int64_t row = row0 + threadIdx.x / TPR;
        if (TPR <= 64 && row >= a.n) break;
        const T* const dy = (const T*)a.dy + row * a.dy_stride;
        const T* const h = (const T*)a.h + row * a.h_stride;
        const T* const in = a.dh_in ? (const T*)a.dh_in + row * a.dh_in_stride : nullptr;
        T* const dx = (T*)a.dx + row * a.dx_stride;
        float g[K][N], x[K][N];
        typename Pack<T, N>::V more[K];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll K
        for (int k = 0; k < (KEEP ? KEEP : vectors); ++k) {
            const NormVector q = vector(k);
            const int b = KEEP ? k : 0;
            if (q.in) {
                load_some<END>(g[b], dy + q.col, a.dim - q.col);
                load_some<END>(x[b], h + q.col, a.dim - q.col);
                if (END == OVER && in) more[b] = *reinterpret_cast<const typename Pack<T, N>::V*>(in + q.col);
                if (!KEEP) load_weight<END, T>(w[0], a.weight, a.weight_f32, q.col, a.dim - q.col);
            } else
#pragma unroll
                for (int e = 0; e < N; ++e) g[b][e] = x[b][e] = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                s1 = counts<END>(q, e) ? fmaf(g[b][e] * w[b][e], x[b][e], s1) : s1;
                s2 = counts<END>(q, e) ? fmaf(x[b][e], x[b][e], s2) : s2;
            }
        }
        if (END == OVER && TPR <= 64) read_before_stores();
        row_sums<TPR>(s1, s2, lds + turn);
        const float rho = rsqrtf(s2 / (float)a.dim + a.eps), m = rho * rho * (s1 / (float)a.dim);
#pragma unroll K
        for (int k = 0; k < (KEEP ? KEEP : vectors); ++k) {
            const NormVector q = vector(k);
            const int b = KEEP ? k : 0, live = a.dim - q.col;
            if (!q.in) continue;
            if (!KEEP) {
                load_some<END>(g[0], dy + q.col, live);
                load_some<END>(x[0], h + q.col, live);
                load_weight<END, T>(w[0], a.weight, a.weight_f32, q.col, live);
                load_some<END>(dw[0], part + q.col, live);
            }
            float o[N];
            if (END != OVER && in) load_some<END>(o, in + q.col, live);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                dw[b][e] = fmaf(g[b][e], x[b][e] * rho, dw[b][e]);
                const float t = rho * (g[b][e] * w[b][e] - x[b][e] * m);
                o[e] = in ? (END == OVER ? (float)more[b][e] : o[e]) + t : t;
            }
            store_some<END>(dx + q.col, o, live);
            if (!KEEP) store_some<END>(part + q.col, dw[0], live);
        }
    }
    // (columns that two lanes have: both have added the same numbers up, in the same order)
    if constexpr (KEEP > 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const NormVector q = vector(k);
            if constexpr (GROUPS == 1) { if (q.in) store_some<END>(part + q.col, dw[k], a.dim - q.col); }
            else if (q.in)
#pragma unroll
                for (int e = 0; e < N; ++e) cols[threadIdx.x / TPR * (TPR * K * N) + q.col + e] = dw[k][e];
        }
        if constexpr (GROUPS > 1) {
            __syncthreads();
            for (int col = threadIdx.x; col < a.dim; col += NT) {
                float s = 0.f;
                for (int gr = 0; gr < GROUPS; ++gr) s += cols[gr * (TPR * K * N) + col];
                part[col] = s;
            }
        }
    }
}

// Columns of the workgroups' sums added up: 64 columns a workgroup, each by 16 threads that take the rows in turn.
constexpr int DW_COLS = 64, DW_PARTS = 16;
template <class W>
__global__ __launch_bounds__(DW_COLS * DW_PARTS) void k_norm_dw(const float* __restrict__ part, int rows, int dim, W* __restrict__ dw) {
    __shared__ float lds[DW_PARTS][DW_COLS];
    const int c = threadIdx.x % DW_COLS, p = threadIdx.x / DW_COLS, col = blockIdx.x * DW_COLS + c;
    float s = 0.f;
    if (col < dim) {
#pragma unroll 8
        for (int r = p; r < rows; r += DW_PARTS) s += part[(size_t)r * dim + col];
    }
    lds[p][c] = s;
    __syncthreads();
    if (p == 0 && col < dim) {
        s = 0.f;
#pragma unroll
        for (int k = 0; k < DW_PARTS; ++k) s += lds[k][c];
        dw[col] = (W)s;
    }
}

// Workgroups of the backward pass, each with a row of sums.  us a call, 256 / 512 / 1024 / 2048 at most (16-bit rows with the residual's gradient): 16,384 rows of 4096
// columns 207 / 127 / 106 / 112, 4096 57 / 38 / 36 / 42, 1024 15.1 / 14.4 / 17.8 / 17.8, 8192 of 8192 151 / 104 / 112 / 127, 16,384 of 1024 65 / 42 / 33 / 37,
// 400 k of 256 330 / 194 / 155 / 169.  (Up to a few thousand rows the sums are as many bytes as the rows, and fewer workgroups would do.)
constexpr int NORM_BWD_BLOCKS = 1024;
// Rows of sums: one a workgroup, of which there are no more than rows.  Up to 32 MB (8192 columns) there is room for all of them, so that the workspace does
// not grow, and the call that grows it does not wait, each time a call has more rows than those before.
size_t norm_work_bytes(int64_t n, int64_t dim) {
    const size_t row = (size_t)dim * 4;
    return std::max(std::min(NORM_BWD_BLOCKS * row, (size_t)32 << 20), (size_t)std::min<int64_t>(n, NORM_BWD_BLOCKS) * row);
}

// f(shape): lanes of a row, vectors a lane keeps, what its last vector is.  Up to a wavefront a row's lanes are as many as its vectors.
// Wider rows: a vector to a lane where there are few of them (`few`), which then wait for nothing but one round of loads; else more of them to a
// lane, and fewer lanes.
template <int TPR_, int KEEP_, int END_> struct NormShape { static constexpr int TPR = TPR_, KEEP = KEEP_, END = END_; };
// us a launch, one vector / more of them (16-bit rows with residual): 4096 columns, 1 row 2.5 / 3.0, 256 rows 3.3 / 3.8, 512 4.3 / 4.7, 1024 7.6 / 7.7, 2048
// 12.0 / 11.7, 8192 49 / 53; 8192 columns, 1 row 2.8 / 4.2, 256 rows 4.4 / 5.9, 512 7.6 / 8.5, 1024 12.5 / 12.2, 2048 29.1 / 26.5, 8192 99.7 / 105.
constexpr int64_t NORM_FEW = 512;                  // rows
template <int N, class F>
static void norm_shape(int dim, bool few, F f) {
    const int64_t vectors = cdiv(dim, N);
    auto kept = [&](auto end) {
        constexpr int E = decltype(end)::value;
        if (vectors <= 8) f(NormShape<8, 1, E>());
        else if (vectors <= 16) f(NormShape<16, 1, E>());
        else if (vectors <= 32) f(NormShape<32, 1, E>());
        else if (vectors <= 64) f(NormShape<64, 1, E>());
        else if (vectors <= 128 && !few) f(NormShape<64, 2, E>());
        else if (vectors <= 256) f(NormShape<256, 1, E>());
        else if (vectors <= 512 && few) f(NormShape<512, 1, E>());
        else if (vectors <= 1024 && few) f(NormShape<1024, 1, E>());
        else if (vectors <= 512) f(NormShape<256, 2, E>());
        else if (vectors <= 1024) f(NormShape<256, 4, E>());
        else f(NormShape<1024, 4, E>());
    };
    if (dim < N) f(NormShape<8, 1, PART>());
    else if (vectors > 4096) f(NormShape<1024, 0, PART>());
    else if (dim % N) kept(std::integral_constant<int, OVER>());
    else kept(std::integral_constant<int, WHOLE>());
}

// The backward pass keeps three rows, the weights and the weights' gradient: half as many vectors a lane (four: 202 registers, and with 1024 threads
// they spill).
template <int N, class F>
static void norm_bwd_shape(int dim, F f) {
    const int64_t vectors = cdiv(dim, N);
    auto kept = [&](auto end) {
        constexpr int E = decltype(end)::value;
        if (vectors <= 8) f(NormShape<8, 1, E>());
        else if (vectors <= 16) f(NormShape<16, 1, E>());
        else if (vectors <= 32) f(NormShape<32, 1, E>());
        else if (vectors <= 64) f(NormShape<64, 1, E>());
        else if (vectors <= 128) f(NormShape<64, 2, E>());
        else if (vectors <= 256) f(NormShape<256, 1, E>());
        else if (vectors <= 512) f(NormShape<256, 2, E>());
        else if (vectors <= 1024) f(NormShape<512, 2, E>());
        else f(NormShape<1024, 2, E>());
    };
    if (dim < N) f(NormShape<8, 1, PART>());
    else if (vectors > 2048) f(NormShape<1024, 0, PART>());
    else if (dim % N) kept(std::integral_constant<int, OVER>());
    else kept(std::integral_constant<int, WHOLE>());
}

}  // namespace fc

using namespace fc;

extern "C" {

int rms_norm_fwd(fc_dense* d, const void* x_dev, int32_t type, int64_t x_stride, const void* residual_dev, int64_t residual_stride, const void* weight_dev,
                 int32_t weight_type, int64_t n, int32_t dim, float eps, void* h_dev, int64_t h_stride, void* y_dev, int32_t y_type, int64_t y_stride,
                 float* scales_dev, int32_t group) {
    const bool quant = y_type == FC_TYPE_F8E4M3 || y_type == FC_TYPE_I8;
    if (!d || n < 0 || n >= DENSE_LIMIT || dim <= 0 || dim > DENSE_MAX_DIM || !is_float_type(type) || (weight_type != FC_TYPE_F32 && weight_type != type) ||
        (!quant && y_type != type) || (quant ? group != 0 && group != 32 && group != 64 && group != 128 && group != 256 : group != 0) ||
        !(eps >= 0.f) || x_stride < dim || (residual_dev && residual_stride < dim) || (h_dev && h_stride < dim) || y_stride < dim || !weight_dev ||
        (n > 0 && (!x_dev || !y_dev || (quant && !scales_dev))))
        return FC_ERR_INVALID_ARG;
    if (n == 0) return FC_OK;
    FC_HIP(hipSetDevice(d->device));
    NormFwd a{x_dev, residual_dev, weight_dev, h_dev, y_dev, scales_dev, x_stride, residual_stride, h_stride, y_stride, 0, n, dim,
                    weight_type == FC_TYPE_F32, group, eps};
    return with_type(type, [&](auto t) -> int {
        using T = decltype(t);
        norm_shape<VECTOR<T>>(dim, n < NORM_FEW, [&](auto s) {
            using S = decltype(s);
            constexpr int NT = norm_threads(S::TPR);
            constexpr int64_t MOST = LAUNCH_THREADS / S::TPR;             // (a multiple of a workgroup's rows)
            for (; a.first < n; a.first += MOST) {
                const unsigned blocks = (unsigned)cdiv(std::min(MOST, n - a.first), NT / S::TPR);
                if (y_type == FC_TYPE_F8E4M3) k_norm_fwd<S::TPR, S::KEEP, S::END, T, F8><<<blocks, NT, 0, d->stream>>>(a);
                else if (y_type == FC_TYPE_I8) k_norm_fwd<S::TPR, S::KEEP, S::END, T, int8_t><<<blocks, NT, 0, d->stream>>>(a);
                else k_norm_fwd<S::TPR, S::KEEP, S::END, T, T><<<blocks, NT, 0, d->stream>>>(a);
            }
        });
        FC_HIP(hipGetLastError());
        return FC_OK;
    });
}

int rms_norm_bwd(fc_dense* d, const void* grad_y_dev, int64_t grad_y_stride, const void* h_dev, int32_t type, int64_t h_stride, const void* weight_dev,
                 int32_t weight_type, const void* grad_h_dev, int64_t grad_h_stride, int64_t n, int32_t dim, float eps, void* grad_x_dev,
                 int64_t grad_x_stride, void* grad_weight_dev, int32_t grad_weight_type) {
    if (!d || n < 0 || n >= DENSE_LIMIT || dim <= 0 || dim > DENSE_MAX_DIM || !is_float_type(type) || (weight_type != FC_TYPE_F32 && weight_type != type) ||
        !is_float_type(grad_weight_type) || !(eps >= 0.f) || grad_y_stride < dim || h_stride < dim || (grad_h_dev && grad_h_stride < dim) ||
        grad_x_stride < dim || !weight_dev || !grad_weight_dev || (n > 0 && (!grad_y_dev || !h_dev || !grad_x_dev)))
        return FC_ERR_INVALID_ARG;
    FC_HIP(hipSetDevice(d->device));
    FC_TRY(dense_work(d, norm_work_bytes(n, dim)));
    float* part = reinterpret_cast<float*>(d->work);
    const NormBwd a{grad_y_dev, h_dev, weight_dev, grad_h_dev, grad_x_dev, part, grad_y_stride, h_stride, grad_h_stride, grad_x_stride, n, dim,
                    weight_type == FC_TYPE_F32, eps};
    int64_t blocks = 0;
    const int rc = with_type(type, [&](auto t) -> int {
        using T = decltype(t);
        if (n > 0) norm_bwd_shape<VECTOR<T>>(dim, [&](auto s) {
            using S = decltype(s);
            constexpr int NT = norm_threads(S::TPR);
            blocks = std::min<int64_t>(cdiv(n, NT / S::TPR), NORM_BWD_BLOCKS);
            k_norm_bwd<S::TPR, S::KEEP, S::END, T><<<(unsigned)blocks, NT, 0, d->stream>>>(a);
        });
        FC_HIP(hipGetLastError());
        return FC_OK;
    });
    if (rc != FC_OK) return rc;
    return with_type(grad_weight_type, [&](auto t) -> int {
        using W = decltype(t);
        k_norm_dw<<<(unsigned)cdiv(dim, DW_COLS), DW_COLS * DW_PARTS, 0, d->stream>>>(part, (int)blocks, dim, (W*)grad_weight_dev);
        FC_HIP(hipGetLastError());
        return FC_OK;
    });
}

}  // extern "C"
