// Distillation from a teacher's top logits, with cross entropy beside it: the loss of each row, and the gradient of its logits.
//
//   row of logits x[0 .. V), entries (t_k, z_k) of the teacher, temperature T, a = alpha, target y
//   P_k = exp(z_k / T - L), L the teacher's log-sum over all ids if it is known (then P_0 = max(0, 1 - sum P_k) is what the entries leave over), else over
//   its entries (P_0 = 0);  Q = softmax(x / T), Q_0 = the sum of Q over the ids that no entry names
//   loss   = a T^2 [sum P_k (log P_k - log Q[t_k]) + P_0 (log P_0 - log Q_0)] + (1 - a) [-log softmax(x)[y]]
//   d/dx_v = a T [c Q_v - sum of P_k with t_k = v] + (1 - a) [softmax(x)_v - (v = y)] for a named v, c = sum P_k + P_0
//            a T [c Q_v - P_0 Q_v / Q_0]           + (1 - a) [softmax(x)_v - (v = y)] for the others
//
// A slice of a row is in registers, so each pass reads the logits once: HBM bounds it.  With P_0 the sums over the ids that are not named are kept apart from those
// over the named ones, each relative to its own largest element, so that neither is a difference of nearly equal numbers nor lost below the other.
// The gradient of the others is then one product with an exponential; the entries and the target are mended afterwards, from their own formula.
#include "logits_device.h"

#include <algorithm>

#include <type_traits>

namespace fc {

constexpr int DISTILL_MAX_TOP = 1024;
constexpr int STATS = 12;                          // numbers of a row that the forward pass leaves for the backward pass
enum { ST_OFF, ST_COEF, ST_OFF1, ST_COEF1, ST_ALL, ST_INV, ST_ALL1, ST_INV1, ST_NAMED, ST_ZFROM, ST_ZINV, ST_KIND };
// ST_KIND
constexpr float ROW_OUT = 0.f, ROW_TARGET_ONLY = 1.f, ROW_ENTRIES = 2.f;

struct DistillArgs {
    const void* x;                                 // logits
    int64_t stride;
    const void* ids;
    const void* z;
    const float* lse;
    const void* target;
    int64_t n;
    int32_t dim, top, id_type, z_type, target_type;
    float temperature, alpha;
    uint32_t* flags;
};

__device__ __forceinline__ float scale_of(const DistillArgs& a) { return (float)(1.4426950408889634 / (double)a.temperature); }
__device__ __forceinline__ int64_t load_id(const void* p, int type, int64_t i) {
    return type == FC_TYPE_I64 ? ((const int64_t*)p)[i] : (int64_t)((const int32_t*)p)[i];
}
__device__ __forceinline__ float load_value(const void* p, int type, int64_t i) {
    return type == FC_TYPE_F32 ? ((const float*)p)[i] : type == FC_TYPE_BF16 ? (float)((const bf16*)p)[i] : (float)((const f16*)p)[i];
}
// an id of the vocabulary, or -1; those outside raise the sticky error
__device__ __forceinline__ int known_id(int64_t id, int dim, uint32_t* flags) {
    if (id >= 0 && id < dim) return (int)id;
    if (id != -1) atomicOr(flags, (uint32_t)EF_ID_RANGE);
    return -1;
}
// The row's target; false if the row is left out.
__device__ __forceinline__ bool row_target(const DistillArgs& a, int64_t row, int* y) {
    *y = -1;
    if (!a.target) return true;
    *y = known_id(load_id(a.target, a.target_type, row), a.dim, a.flags);
    return *y >= 0;
}

// Sums of exponentials at the temperature and at 1: t = sum of 2^(x ct - off), ct = log2(e) / T rounded to 32 bits; one = sum of 2^(x log2(e) - off1).  The offsets are the
// rounded products of the largest element, and what is joined or taken further goes by the offsets, so that their rounding cancels (2e-6 of
// each exponential for logits of 30 otherwise), and so does that of ct but for its share in differences from the largest.
struct Sums {
    float off, off1, t, one;
    __device__ __forceinline__ void join(const Sums& o) {
        const float most = fmaxf(off, o.off), most1 = fmaxf(off1, o.off1), to = from_of(most), to1 = from_of(most1);
        t = t * __builtin_amdgcn_exp2f(off - to) + o.t * __builtin_amdgcn_exp2f(o.off - to);
        one = one * __builtin_amdgcn_exp2f(off1 - to1) + o.one * __builtin_amdgcn_exp2f(o.off1 - to1);
        off = most;
        off1 = most1;
    }
    __device__ __forceinline__ Sums over_wave() const {
        Sums s;
        s.off = wave_max(off);
        s.off1 = wave_max(off1);
        s.t = wave_sum(t * __builtin_amdgcn_exp2f(off - from_of(s.off)));
        s.one = wave_sum(one * __builtin_amdgcn_exp2f(off1 - from_of(s.off1)));
        return s;
    }
};
constexpr double LN2 = 0.69314718055994530942;
constexpr Sums NO_SUMS{-INFINITY, -INFINITY, 0.f, 0.f};
struct RowSums { Sums rest, named; };

// What a wavefront makes of a row's sums: its loss and, if wanted, the numbers for the backward pass.
template <class T>
__device__ void distill_row(const DistillArgs& a, int64_t row, int y, const RowSums& s, float* __restrict__ loss, float* __restrict__ stats) {
    const int lane = threadIdx.x & 63;
    const T* x = (const T*)a.x + row * a.stride;
    const double it = 1.0 / (double)a.temperature;
    const float ct = scale_of(a), it32 = (float)it;
    Sums all = s.rest;
    all.join(s.named);
    const double lse2 = (double)all.off + (double)log2f(all.t);

    float zmax = -INFINITY;
    bool some = false;
    for (int k = lane; k < a.top; k += 64) {
        const int64_t i = row * a.top + k;
        if (known_id(load_id(a.ids, a.id_type, i), a.dim, a.flags) < 0) continue;
        const float z = load_value(a.z, a.z_type, i);
        zmax = fmaxf(zmax, z);
        some |= a.lse || z != -INFINITY;
    }
    some = __any(some);
    zmax = from_of(wave_max(zmax));
    float kl = 0.f, part = 0.f, zinv = 0.f, sum_p = 0.f, p0 = 0.f, q0 = 1.f;
    if (some && a.alpha > 0.f) {
        double log_zinv;
        if (a.lse) {
            log_zinv = (double)zmax * it - (double)a.lse[row];
            zinv = expf((float)log_zinv);
        } else {
            float sum = 0.f;
            for (int k = lane; k < a.top; k += 64) {
                const int64_t i = row * a.top + k;
                const int64_t id = load_id(a.ids, a.id_type, i);
                if (id >= 0 && id < a.dim) sum += expf((load_value(a.z, a.z_type, i) - zmax) * it32);
            }
            sum = wave_sum(sum);
            zinv = 1.f / sum;
            log_zinv = -(double)logf(sum);
        }
        for (int k = lane; k < a.top; k += 64) {
            const int64_t i = row * a.top + k;
            const int64_t id = load_id(a.ids, a.id_type, i);
            if (id < 0 || id >= a.dim) continue;
            const double d = ((double)load_value(a.z, a.z_type, i) - zmax) * it;
            const float p = expf((float)d) * zinv;
            part += p;
            if (p == 0.f) continue;                // nothing, also where the student gives nothing
            const double log_q = ((double)(float)x[id] * ct - lse2) * LN2;
            kl += p * (float)(d + log_zinv - log_q);
        }
        kl = wave_sum(kl);
        sum_p = wave_sum(part);
        if (a.lse) {
            p0 = fmaxf(0.f, 1.f - sum_p);
            const double log_q0 = ((double)s.rest.off + (double)log2f(s.rest.t) - lse2) * LN2;
            q0 = expf((float)log_q0);
            if (p0 > 0.f) kl += p0 * (logf(p0) - (float)log_q0);
        }
    }
    if (lane != 0) return;
    float value = some && a.alpha > 0.f ? a.alpha * a.temperature * a.temperature * kl : 0.f;
    if (a.alpha < 1.f) value += (1.f - a.alpha) * (float)(((double)all.off1 + (double)log2f(all.one) - (double)(float)x[y] * LOG2E) * LN2);
    if (loss) loss[row] = value;
    if (!stats) return;
    float* o = stats + row * STATS;
    const float c = sum_p + p0;
    float coef = 0.f, coef1 = 0.f;
    if (s.rest.t != 0.f) {                         // (else there is nothing that is not named, or only logits of -infinity)
        if (some) coef = a.alpha * a.temperature * (c * q0 - p0) / s.rest.t;
        if (a.alpha < 1.f) coef1 = (1.f - a.alpha) * exp2f(s.rest.off1 - all.off1) / all.one;
    }
    if (all.t == 0.f) coef = NAN;                  // all logits are -infinity
    const bool one = a.temperature == 1.f;         // one exponential stands for both
    o[ST_OFF] = from_of(s.rest.off);
    o[ST_COEF] = one ? coef + coef1 : coef;
    o[ST_OFF1] = from_of(s.rest.off1);
    o[ST_COEF1] = one ? 0.f : coef1;
    o[ST_ALL] = all.off;
    o[ST_INV] = 1.f / all.t;
    o[ST_ALL1] = all.off1;
    o[ST_INV1] = 1.f / all.one;
    o[ST_NAMED] = c;
    o[ST_ZFROM] = zmax;
    o[ST_ZINV] = zinv;
    o[ST_KIND] = some && a.alpha > 0.f ? ROW_ENTRIES : a.alpha < 1.f ? ROW_TARGET_ONLY : ROW_OUT;
}

__device__ __forceinline__ void distill_left_out(int64_t row, float* loss, float* stats) {
    if ((threadIdx.x & 63) >= STATS) return;
    if ((threadIdx.x & 63) == 0 && loss) loss[row] = 0.f;
    if (stats) stats[row * STATS + (threadIdx.x & 63)] = 0.f;
}

// Sums of a slice, over LANES lanes of a row.  REST: named ids apart from the others.  `slices` > 1: the sums go to `part`, else the row is finished.
template <class T, int LANES, int PER, bool REST>
__global__ __launch_bounds__(LOGIT_THREADS) void k_distill_fwd(DistillArgs a, int slices, RowSums* __restrict__ part, float* __restrict__ loss, float* __restrict__ stats) {
    using Slice = RowSlice<T, LANES, PER>;
    constexpr int N = Slice::N, ROWS = LOGIT_THREADS / LANES, WORDS = LANES * PER / 4;
    __shared__ uint32_t marks[REST ? ROWS : 1][REST ? WORDS : 1];      // a byte for each vector, a bit for each element that is named
    __shared__ RowSums lds[LOGIT_THREADS / 64];
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    const int64_t row = (int64_t)(blockIdx.x / slices) * ROWS + sub;
    const int slice = blockIdx.x % slices, base = slice * Slice::COLUMNS;
    if (row >= a.n) return;                        // (all lanes of the row)
    int y;
    if (!row_target(a, row, &y)) {
        if (slice == 0 && lane < 64) distill_left_out(row, loss, stats);
        return;
    }
    const float ct = scale_of(a);
    const bool two = a.alpha < 1.f && a.temperature != 1.f;
    Slice s;
    s.load((const T*)a.x + row * a.stride, base, lane, a.dim);
    if constexpr (REST) {
#pragma unroll
        for (int k = lane; k < WORDS; k += LANES) marks[sub][k] = 0;
        row_sync<LANES>();
        for (int k = lane; k < a.top; k += LANES) {
            const int64_t id = load_id(a.ids, a.id_type, row * a.top + k) - base;
            if (id >= 0 && id < min(Slice::COLUMNS, a.dim - base)) atomicOr(&marks[sub][id / N / 4], 1u << (id / N % 4 * 8 + id % N));
        }
        row_sync<LANES>();
    }
    auto marked = [&](int k) -> uint32_t {         // of vector k, in the order of its elements as they are loaded
        const int v = k * LANES + lane;
        return (uint32_t)reinterpret_cast<const uint8_t*>(marks[sub])[v] << Slice::skip(Slice::column(base, lane, k), a.dim);
    };
    RowSums r;
    r.named = NO_SUMS;
    float top = -INFINITY, top_named = -INFINITY;
    if constexpr (REST) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t b = marked(k);
            if (b == 0) {
#pragma unroll
                for (int e = 0; e < N; ++e) top = fmaxf(top, s.at(k, e));
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float v = s.at(k, e);
                    if (b >> e & 1) top_named = fmaxf(top_named, v); else top = fmaxf(top, v);
                }
            }
        }
    } else top = s.largest();
    auto sum_of = [&](float c, float off, float off_named, float* named) {
        const float by = -from_of(off), by_named = -from_of(off_named);
        float sum = 0.f;
        *named = 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t b = REST ? marked(k) : 0;
            if (!REST || b == 0) {
#pragma unroll
                for (int e = 0; e < N; ++e) sum += __builtin_amdgcn_exp2f(fmaf(s.at(k, e), c, by));
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (b >> e & 1) *named += __builtin_amdgcn_exp2f(fmaf(s.at(k, e), c, by_named));
                    else sum += __builtin_amdgcn_exp2f(fmaf(s.at(k, e), c, by));
                }
            }
        }
        return sum;
    };
    r.rest.off = r.rest.off1 = top * ct;
    if constexpr (REST) r.named.off = r.named.off1 = top_named * ct;
    r.rest.t = r.rest.one = sum_of(ct, r.rest.off, r.named.off, &r.named.t);
    r.named.one = r.named.t;
    if (two) {
        r.rest.off1 = top * LOG2E;
        if constexpr (REST) r.named.off1 = top_named * LOG2E;
        r.rest.one = sum_of(LOG2E, r.rest.off1, r.named.off1, &r.named.one);
    }
    r.rest = r.rest.over_wave();
    if constexpr (REST) r.named = r.named.over_wave();
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = r;
        __syncthreads();
        if (threadIdx.x >= 64) return;
        for (int k = 1; k < LANES / 64; ++k) {
            r.rest.join(lds[k].rest);
            if constexpr (REST) r.named.join(lds[k].named);
        }
    }
    if (slices > 1) { if (lane == 0) part[row * slices + slice] = r; }
    else distill_row<T>(a, row, y, r, loss, stats);
}

// The rows of several slices: a wavefront to a row.
template <class T>
__global__ __launch_bounds__(LOGIT_THREADS) void k_distill_join(DistillArgs a, int slices, const RowSums* __restrict__ part, float* __restrict__ loss, float* __restrict__ stats) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * (LOGIT_THREADS / 64) + threadIdx.x / 64;
    int y;
    if (row >= a.n || !row_target(a, row, &y)) return;
    RowSums r{NO_SUMS, NO_SUMS};
    for (int k = lane; k < slices; k += 64) {
        r.rest.join(part[row * slices + k].rest);
        r.named.join(part[row * slices + k].named);
    }
    r.rest = r.rest.over_wave();
    r.named = r.named.over_wave();
    distill_row<T>(a, row, y, r, loss, stats);
}

// The gradient of a slice.  It may take the place of the logits: a slice is read, its entries among it, before any of it is written.
template <class T, int LANES, int PER>
__global__ __launch_bounds__(LOGIT_THREADS) void k_distill_bwd(DistillArgs a, int slices, const float* __restrict__ grad_loss, int64_t grad_loss_stride,
                                                               const float* __restrict__ stats, T* grad, int64_t grad_stride) {
    using Slice = RowSlice<T, LANES, PER>;
    constexpr int N = Slice::N, ROWS = LOGIT_THREADS / LANES;
    extern __shared__ float dynamic[];             // for each row: ids, probabilities and logits of its entries
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    const int64_t row = (int64_t)(blockIdx.x / slices) * ROWS + sub;
    const int slice = blockIdx.x % slices, base = slice * Slice::COLUMNS;
    if (row >= a.n) return;
    const T* x = (const T*)a.x + row * a.stride;
    T* out = grad + row * grad_stride;
    const float* st = stats + row * STATS;
    const float g = grad_loss[row * grad_loss_stride], kind = st[ST_KIND];
    const int end = min(a.dim, base + Slice::COLUMNS);
    auto store = [&](int k, const float (&v)[N]) {
        const int col = Slice::column(base, lane, k);
        if (col + N <= a.dim) store_vector(out + col, v);
        else {
#pragma unroll
            for (int e = 0; e < N; ++e) {          // v ends with the row
                const int c = a.dim - N + e;
                if (c >= col) out[c] = (T)v[e];
            }
        }
    };
    if (kind == ROW_OUT || g == 0.f) {
        const float zero[N] = {};
#pragma unroll
        for (int k = 0; k < PER; ++k) store(k, zero);
        return;
    }
    int* ids = reinterpret_cast<int*>(dynamic) + (size_t)sub * 3 * a.top;
    float* p = reinterpret_cast<float*>(ids + a.top);
    float* xs = p + a.top;
    const float it = (float)(1.0 / (double)a.temperature), ct = scale_of(a);
    const float off = -st[ST_OFF], off1 = -st[ST_OFF1], coef = g * st[ST_COEF], coef1 = g * st[ST_COEF1];
    const bool two = a.alpha < 1.f && a.temperature != 1.f;
    Slice s;
    s.load(x, base, lane, a.dim);
    const int entries = kind == ROW_ENTRIES ? a.top : 0;
    for (int k = lane; k < entries; k += LANES) {
        const int64_t i = row * a.top + k;
        const int64_t id = load_id(a.ids, a.id_type, i);
        const bool here = id >= base && id < end;
        ids[k] = here ? (int)id : -1;
        if (here) {
            p[k] = expf((load_value(a.z, a.z_type, i) - st[ST_ZFROM]) * it) * st[ST_ZINV];
            xs[k] = (float)x[id];
        }
    }
    int y = -1;
    float xy = 0.f;
    if (a.target && a.alpha < 1.f) {
        y = (int)load_id(a.target, a.target_type, row);
        if (y < base || y >= end) y = -1;
        else xy = (float)x[y];
    }
    row_sync<LANES>();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = coef * __builtin_amdgcn_exp2f(fmaf(s.at(k, e), ct, off));
        if (two) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = fmaf(coef1, __builtin_amdgcn_exp2f(fmaf(s.at(k, e), LOG2E, off1)), v[e]);
        }
        store(k, v);
    }
    row_sync<LANES>();
    const float scale = a.alpha * a.temperature, hard = 1.f - a.alpha;
    bool y_named = false;
    for (int k = lane; k < entries; k += LANES) {
        const int id = ids[k];
        if (id < 0) continue;
        float sum = 0.f;
        bool first = true;
        for (int j = 0; j < entries; ++j)
            if (ids[j] == id) { first &= j >= k; sum += p[j]; }
        y_named |= id == y;
        if (!first) continue;
        const float q = exp2f(fmaf(xs[k], ct, -st[ST_ALL])) * st[ST_INV], q1 = a.alpha < 1.f ? exp2f(fmaf(xs[k], LOG2E, -st[ST_ALL1])) * st[ST_INV1] : 0.f;
        out[id] = (T)(g * (scale * (st[ST_NAMED] * q - sum) + hard * (q1 - (id == y ? 1.f : 0.f))));
    }
    if (y >= 0) {                                  // (the same in all lanes of the row)
        if constexpr (LANES > 64) y_named = __syncthreads_or(y_named);
        else y_named = __any(y_named);
        if (!y_named && lane == 0) {
            float v = coef * __builtin_amdgcn_exp2f(fmaf(xy, ct, off));
            if (two) v = fmaf(coef1, __builtin_amdgcn_exp2f(fmaf(xy, LOG2E, off1)), v);
            out[y] = (T)(v - g * hard);
        }
    }
}

// Row-slices of one launch: what their sums take of the workspace, and what a launch can have of workgroups, is bounded; more rows go in several.
constexpr int64_t DISTILL_SLICES = 1 << 16;
constexpr size_t DISTILL_WORK = DISTILL_SLICES * (sizeof(RowSums) + STATS * sizeof(float));
size_t distill_work_bytes() { return DISTILL_WORK; }

// f(lanes of a slice, vectors of a lane), as constants, for n rows of `vectors`
template <class F>
void by_slice(int64_t n, int64_t vectors, F f) {
    using std::integral_constant;
    if (vectors <= 64 * 2) f(integral_constant<int, 64>(), integral_constant<int, 2>());
    else if (vectors <= 64 * 8) f(integral_constant<int, 64>(), integral_constant<int, 8>());
    else if (n * cdiv(vectors, LOGIT_THREADS * 8) < 512) f(integral_constant<int, 256>(), integral_constant<int, 2>());
    else f(integral_constant<int, 256>(), integral_constant<int, 8>());
}

// the rows [at, at + n) of a call
static DistillArgs rows_of(const DistillArgs& a, int64_t at, int64_t n, int elem) {
    DistillArgs b = a;
    auto by = [](const void* p, int64_t bytes) { return p ? (const char*)p + bytes : nullptr; };
    auto id_bytes = [](int t) { return t == FC_TYPE_I64 ? 8 : 4; };
    b.x = by(a.x, at * a.stride * elem);
    b.ids = by(a.ids, at * a.top * id_bytes(a.id_type));
    b.z = by(a.z, at * a.top * type_bytes(a.z_type));
    b.lse = a.lse ? a.lse + at : nullptr;
    b.target = by(a.target, at * id_bytes(a.target_type));
    b.n = n;
    return b;
}

struct DistillCall {
    fc_dense* d;
    DistillArgs a;
    const float* grad_loss;
    int64_t grad_loss_stride;
    float *loss, *stats;                           // stats: NULL, then those of a part of the rows are in the workspace if the backward pass follows
    void* grad;
    int64_t grad_stride;
    bool fwd, bwd;
};

template <class T>
int distill_run(const DistillCall& c) {
    constexpr int N = VECTOR<T>;
    const DistillArgs& a = c.a;
    const hipStream_t st = c.d->stream;
    if (c.fwd) FC_TRY(dense_work(c.d, DISTILL_WORK));
    RowSums* part = reinterpret_cast<RowSums*>(c.d->work);
    float* work_stats = reinterpret_cast<float*>(c.d->work + DISTILL_SLICES * sizeof(RowSums));
    by_slice(a.n, cdiv(a.dim, N), [&](auto l, auto p) {
        constexpr int LANES = decltype(l)::value, PER = decltype(p)::value, ROWS = LOGIT_THREADS / LANES;
        const int slices = (int)cdiv(a.dim, RowSlice<T, LANES, PER>::COLUMNS);
        const int64_t most = DISTILL_SLICES / slices;
        for (int64_t at = 0; at < a.n; at += most) {
            const int64_t n = std::min(most, a.n - at);
            const DistillArgs b = rows_of(a, at, n, sizeof(T));
            float* loss = c.loss ? c.loss + at : nullptr;
            float* stats = c.stats ? c.stats + at * STATS : c.bwd ? work_stats : nullptr;
            const unsigned blocks = (unsigned)(cdiv(n, ROWS) * slices);
            if (c.fwd) {
                if (a.lse && a.alpha > 0.f) k_distill_fwd<T, LANES, PER, true><<<blocks, LOGIT_THREADS, 0, st>>>(b, slices, part, loss, stats);
                else k_distill_fwd<T, LANES, PER, false><<<blocks, LOGIT_THREADS, 0, st>>>(b, slices, part, loss, stats);
                if (slices > 1) k_distill_join<T><<<(unsigned)cdiv(n, LOGIT_THREADS / 64), LOGIT_THREADS, 0, st>>>(b, slices, part, loss, stats);
            }
            if (c.bwd)
                k_distill_bwd<T, LANES, PER><<<blocks, LOGIT_THREADS, (size_t)ROWS * a.top * 12, st>>>(
                    b, slices, c.grad_loss + at * c.grad_loss_stride, c.grad_loss_stride, stats, (T*)c.grad + at * c.grad_stride, c.grad_stride);
        }
    });
    FC_HIP(hipGetLastError());
    return FC_OK;
}

static bool is_id_type(int32_t t) { return t == FC_TYPE_I32 || t == FC_TYPE_I64; }

static int distill_call(const DistillCall& c, int32_t type) {
    const DistillArgs& a = c.a;
    if (!c.d || a.n < 0 || a.n >= DENSE_LIMIT || a.dim <= 0 || a.dim > DENSE_MAX_DIM || a.stride < a.dim || !is_float_type(type) || a.top < 0 || a.top > DISTILL_MAX_TOP ||
        !is_id_type(a.id_type) || !is_float_type(a.z_type) || !is_id_type(a.target_type) || !(a.temperature >= 1.f / 1024 && a.temperature <= 1024.f) || !(a.alpha >= 0.f && a.alpha <= 1.f) ||
        (a.alpha < 1.f && a.n > 0 && !a.target) || (a.n > 0 && !a.x) || (a.n > 0 && a.top > 0 && (!a.ids || !a.z)))
        return FC_ERR_INVALID_ARG;
    if (c.bwd && (c.grad_stride < a.dim || (c.grad_loss_stride != 0 && c.grad_loss_stride != 1) || (a.n > 0 && (!c.grad_loss || !c.grad)) ||
                  (c.grad == a.x && c.grad_stride != a.stride)))
        return FC_ERR_INVALID_ARG;
    if (a.n == 0) return FC_OK;
    FC_HIP(hipSetDevice(c.d->device));
    return with_type(type, [&](auto t) -> int { return distill_run<decltype(t)>(c); });
}

}  // namespace fc

using namespace fc;

extern "C" {

int distill_fwd(fc_dense* d, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t n, int32_t dim, const void* teacher_ids_dev, int32_t id_type,
                const void* teacher_dev, int32_t teacher_type, int32_t top, const float* teacher_lse_dev, const void* targets_dev, int32_t target_type,
                float temperature, float alpha, float* loss_dev, float* stats_dev) {
    if (!d || (n > 0 && (!loss_dev || !stats_dev))) return FC_ERR_INVALID_ARG;
    DistillCall c{};
    c.d = d;
    c.a = DistillArgs{logits_dev, logits_stride, teacher_ids_dev, teacher_dev, teacher_lse_dev, targets_dev, n, dim, top, id_type, teacher_type, target_type, temperature, alpha, d->flags};
    c.loss = loss_dev; c.stats = stats_dev; c.fwd = true;
    return distill_call(c, type);
}

int distill_bwd(fc_dense* d, const float* grad_loss_dev, int64_t grad_loss_stride, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t n, int32_t dim,
                const void* teacher_ids_dev, int32_t id_type, const void* teacher_dev, int32_t teacher_type, int32_t top, const void* targets_dev, int32_t target_type,
                float temperature, float alpha, const float* stats_dev, void* grad_logits_dev, int64_t grad_logits_stride) {
    if (!d || (n > 0 && !stats_dev)) return FC_ERR_INVALID_ARG;
    DistillCall c{};
    c.d = d;
    c.a = DistillArgs{logits_dev, logits_stride, teacher_ids_dev, teacher_dev, nullptr, targets_dev, n, dim, top, id_type, teacher_type, target_type, temperature, alpha, d->flags};
    c.grad_loss = grad_loss_dev; c.grad_loss_stride = grad_loss_stride; c.stats = const_cast<float*>(stats_dev);
    c.grad = grad_logits_dev; c.grad_stride = grad_logits_stride; c.bwd = true;
    return distill_call(c, type);
}

int distill_grad(fc_dense* d, const float* grad_loss_dev, int64_t grad_loss_stride, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t n, int32_t dim,
                 const void* teacher_ids_dev, int32_t id_type, const void* teacher_dev, int32_t teacher_type, int32_t top, const float* teacher_lse_dev,
                 const void* targets_dev, int32_t target_type, float temperature, float alpha, float* loss_dev, void* grad_logits_dev, int64_t grad_logits_stride) {
    if (!d || (n > 0 && !loss_dev)) return FC_ERR_INVALID_ARG;
    DistillCall c{};
    c.d = d;
    c.a = DistillArgs{logits_dev, logits_stride, teacher_ids_dev, teacher_dev, teacher_lse_dev, targets_dev, n, dim, top, id_type, teacher_type, target_type, temperature, alpha, d->flags};
    c.grad_loss = grad_loss_dev; c.grad_loss_stride = grad_loss_stride; c.loss = loss_dev;
    c.grad = grad_logits_dev; c.grad_stride = grad_logits_stride; c.fwd = c.bwd = true;
    return distill_call(c, type);
}

}  // extern "C"
