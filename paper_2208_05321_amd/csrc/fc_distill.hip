// Distillation from a teacher's top logits, with cross entropy beside it: the loss of each row, and the gradient of its logits.
//
//   row of logits x[0 .. V), entries (t_k, z_k) of the teacher, temperature T, a = alpha, target y
//   P_k = exp(z_k / T - L), L the teacher's log-sum over all ids if it is known (then P_0 = max(0, 1 - sum P_k) is what the entries leave over), else over
//   its entries (P_0 = 0);  Q = softmax(x / T), Q_0 = the sum of Q over the ids that no entry names
//   loss   = a T^2 [sum P_k (log P_k - log Q[t_k]) + P_0 (log P_0 - log Q_0)] + (1 - a) [-log softmax(x)[y]]
//   d/dx_v = a T [c Q_v - sum of P_k with t_k = v] + (1 - a) [softmax(x)_v - (v = y)] for a named v, c = sum P_k + P_0
//            a T [c Q_v - P_0 Q_v / Q_0]           + (1 - a) [softmax(x)_v - (v = y)] for the others
//
// A slice of a row is in registers, so each pass reads the logits once: HBM bounds it.  Times of calls: 8192 rows of 131,072 bf16, loss: 330 us, 6.5 TB/s; loss and gradient together of
// 16,384 rows of 32,768, each read once and written once: 412 us, 5.2 TB/s (rows wait in registers for their sums); of 4096 rows of 131,072 in two passes 560 us, of which the second kernel 356, 6.0 TB/s.  With P_0 the sums over the ids that are not named are kept apart from those
// over the named ones, each relative to its own largest element, so that neither is a difference of nearly equal numbers nor lost below the other.
// The gradient of the others is then one product with an exponential; the entries and the target are mended afterwards, from their own formula.
#include "logits_device.h"

#include <algorithm>
#include <type_traits>

namespace fc {

constexpr int DISTILL_MAX_TOP = 1024;
constexpr int STATS = 12;                          // numbers of a row that the forward pass leaves for the backward pass
enum { ST_REST, ST_COEF, ST_COEF1, ST_ALL, ST_INV, ST_INV1, ST_NAMED, ST_ZFROM, ST_ZINV, ST_KIND };      // (and two zeros)
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

// Sums of exponentials at the temperature and at 1, from an element of the logits: t = sum of 2^(ct (x - from)), ct = log2(e) / T rounded to 32 bits, and one = sum of 2^(log2(e) (x - from)).  What the
// rounding of ct makes is in proportion to differences from the largest element, not to the logits; without `two` (the sums at 1 are others than those at the temperature) one is t.
struct Sums {
    float from, t, one;
    __device__ __forceinline__ void join(const Sums& o, float ct, bool two) {
        const float most = fmaxf(from, o.from);
        if (two) one = one * part_of(from, most, LOG2E) + o.one * part_of(o.from, most, LOG2E);
        t = t * part_of(from, most, ct) + o.t * part_of(o.from, most, ct);
        if (!two) one = t;
        from = most;
    }
    // over the wavefront's lanes
    __device__ __forceinline__ Sums over_wave(float ct, bool two) const {
        Sums s;
        s.from = wave_max(from);
        s.t = s.one = wave_sum(t * part_of(from, s.from, ct));
        if (two) s.one = wave_sum(one * part_of(from, s.from, LOG2E));
        return s;
    }
};
constexpr double LN2 = 0.69314718055994530942;
constexpr Sums NO_SUMS{-INFINITY, 0.f, 0.f};
// What is left of a row, or of a slice, without the named ids where P_0 needs that; twice: an id was seen to be named more than once.
struct RowSums { Sums rest; float twice; };

// of an entry's probability, from that of the largest
__device__ __forceinline__ double exponent(float z, float zmax, double it) { return ((double)z - zmax) * it; }

// Entries of a row in LDS: ids (-1: none that counts), the teacher's logits, and later probabilities, the student's logits.
struct Entries { int* id; float* z; float* x; };
constexpr __host__ __device__ int entries_room(int top) { return (top + 3) & ~3; }        // (ids are looked through four at a time)
__device__ __forceinline__ Entries entries_at(float* lds, int sub, int top) {
    const int room = entries_room(top);
    lds += (size_t)sub * 3 * room;
    return Entries{reinterpret_cast<int*>(lds), lds + room, lds + 2 * room};
}
// the places behind the last entry
__device__ __forceinline__ void end_entries(const Entries& t, int lane, int top) { if (top + lane < entries_room(top)) t.id[top + lane] = -1; }
template <class T, int LANES>
__device__ __forceinline__ void load_entries(const DistillArgs& a, int64_t row, int lane, const T* x, const Entries& t) {
    for (int k = lane; k < a.top; k += LANES) {
        const int64_t i = row * a.top + k;
        const float z = load_value(a.z, a.z_type, i);
        const int id = known_id(load_id(a.ids, a.id_type, i), a.dim, a.flags);
        t.id[k] = id;
        t.z[k] = z;
        t.x[k] = id >= 0 ? (float)x[id] : 0.f;
    }
    end_entries(t, lane, a.top);
}

// What a wavefront makes of a row's sums and entries (xy: the target's logit): its loss and the numbers for the backward pass.  The entries' logits become their probabilities.
__device__ __forceinline__ void distill_row(const DistillArgs& a, int64_t row, float xy, const RowSums& s, const Entries& t, float* __restrict__ loss, float* stats) {
    const int lane = threadIdx.x & 63;
    const double it = 1.0 / (double)a.temperature;
    const float ct = scale_of(a);
    const float lse = a.lse ? a.lse[row] : 0.f;
    const bool two = a.alpha < 1.f && a.temperature != 1.f;
    Sums all = s.rest;
    if (a.lse && a.alpha > 0.f) {                  // and the named ones, each once
        Sums named = NO_SUMS;
        for (int k = lane; k < a.top; k += 64) {
            const int id = t.id[k];
            bool counts = id >= 0;
            if (s.twice != 0.f)
                for (int j = 0; j < k; ++j) counts &= t.id[j] != id;
            if (!counts) continue;
            const float x = t.x[k], one = x == -INFINITY ? 0.f : 1.f;
            named.join(Sums{x, one, one}, ct, two);
        }
        all.join(named.over_wave(ct, two), ct, two);
    }
    const float from = from_of(all.from);
    const double log_t = (double)log2f(all.t);

    float zmax = -INFINITY;
    bool some = false;
    for (int k = lane; k < a.top; k += 64) {
        if (t.id[k] < 0) continue;
        const float z = t.z[k];
        zmax = fmaxf(zmax, z);
        some |= a.lse || z != -INFINITY;
    }
    some = a.alpha > 0.f && __any(some);
    zmax = from_of(wave_max(zmax));
    float kl = 0.f, part = 0.f, zinv = 0.f, sum_p = 0.f, p0 = 0.f, q0 = 1.f;
    if (some) {
        double log_zinv;
        if (a.lse) {
            log_zinv = (double)zmax * it - (double)lse;
            zinv = expf((float)log_zinv);
        } else {
            float sum = 0.f;
            for (int k = lane; k < a.top; k += 64)
                if (t.id[k] >= 0) sum += expf((float)exponent(t.z[k], zmax, it));
            sum = wave_sum(sum);
            zinv = 1.f / sum;
            log_zinv = -(double)logf(sum);
        }
        for (int k = lane; k < a.top; k += 64) {
            if (t.id[k] < 0) continue;
            const double d = exponent(t.z[k], zmax, it);
            const float p = expf((float)d) * zinv;
            t.z[k] = p;
            part += p;
            if (p == 0.f) continue;                // nothing, also where the student gives nothing
            const double log_q = (((double)t.x[k] - from) * ct - log_t) * LN2;
            kl += p * (float)(d + log_zinv - log_q);
        }
        kl = wave_sum(kl);
        sum_p = wave_sum(part);
        if (a.lse) {
            p0 = fmaxf(0.f, 1.f - sum_p);
            const double log_q0 = (((double)s.rest.from - from) * ct + (double)log2f(s.rest.t) - log_t) * LN2;
            q0 = expf((float)log_q0);
            // Of a teacher whose entries hold everything P_0 is what roundings leave: of the log-sum, of the exponents and of their sum, half a unit of 32 bits of each, and as much again for a log-sum worked out
            // in 32 bits.  Where the student gives the others nothing that would cost infinitely much, or whatever number masks them.
            if (q0 == 0.f && p0 <= 0x1p-23f * (fabsf(lse) + fabsf((float)log_zinv) + (float)a.top / 64 + 16.f)) p0 = 0.f;
            if (p0 > 0.f) kl += p0 * (logf(p0) - (float)log_q0);
        }
    }
    if (lane != 0) return;
    float value = some ? a.alpha * a.temperature * a.temperature * kl : 0.f;
    if (a.alpha < 1.f) value += (1.f - a.alpha) * (float)((((double)from - xy) * LOG2E + (double)log2f(all.one)) * LN2);
    if (loss) loss[row] = value;
    const float c = sum_p + p0;
    float coef = 0.f, coef1 = 0.f;
    if (s.rest.t != 0.f) {                         // (else there is nothing that is not named, or only logits of -infinity)
        if (some) coef = a.alpha * a.temperature * (c * q0 - p0) / s.rest.t * exponents(s.rest.from, ct).back;
        if (a.alpha < 1.f) coef1 = (1.f - a.alpha) * exp2f((s.rest.from - from) * LOG2E) / all.one * exponents(s.rest.from, LOG2E).back;
    }
    if (all.t == 0.f) coef = NAN;                  // all logits are -infinity
    const bool one = a.temperature == 1.f;         // one exponential stands for both
    stats[ST_REST] = s.rest.from;
    stats[ST_COEF] = one ? coef + coef1 : coef;
    stats[ST_COEF1] = one ? 0.f : coef1;
    stats[ST_ALL] = from;
    stats[ST_INV] = 1.f / all.t;
    stats[ST_INV1] = 1.f / all.one;
    stats[ST_NAMED] = c;
    stats[ST_ZFROM] = zmax;
    stats[ST_ZINV] = zinv;
    stats[ST_KIND] = some ? ROW_ENTRIES : a.alpha < 1.f ? ROW_TARGET_ONLY : ROW_OUT;
    for (int k = ST_KIND + 1; k < STATS; ++k) stats[k] = 0.f;
}

__device__ __forceinline__ void distill_left_out(int64_t row, int lane, float* loss, float* stats) {
    if (lane == 0) loss[row] = 0.f;
    if (lane < STATS && stats) stats[row * STATS + lane] = 0.f;
}

// Marks of a slice's named elements, in LDS: a byte for each vector, those of a lane side by side.
template <int LANES, int PER> struct Marks { uint64_t of[LANES][(PER + 7) / 8]; int32_t twice; };

// Marks the elements of a slice that the row's entries name.
template <class T, int LANES, int PER>
__device__ __forceinline__ void mark_named(const DistillArgs& a, int64_t row, int base, int lane, Marks<LANES, PER>& marks) {
    constexpr int N = VECTOR<T>, COLUMNS = RowSlice<T, LANES, PER>::COLUMNS;
#pragma unroll
    for (int j = 0; j < (PER + 7) / 8; ++j) marks.of[lane][j] = 0;
    if (lane == 0) marks.twice = 0;
    row_sync<LANES>();
    for (int k = lane; k < a.top; k += LANES) {
        const int64_t id = load_id(a.ids, a.id_type, row * a.top + k) - base;
        if (id < 0 || id >= min(COLUMNS, a.dim - base)) continue;
        const int v = (int)id / N, j = v / LANES;
        const uint32_t bit = 1u << (j % 4 * 8 + (int)id % N);
        if (atomicOr(reinterpret_cast<uint32_t*>(&marks.of[v % LANES][0]) + j / 4, bit) & bit) marks.twice = 1;
    }
    row_sync<LANES>();
}

// Adds a slice to a lane's sums; marked elements become -infinity in the registers before.
template <class T, int LANES, int PER>
__device__ __forceinline__ void add_slice(const DistillArgs& a, RowSlice<T, LANES, PER>& s, int base, int lane, const Marks<LANES, PER>* marks, Sums& r) {
    using Slice = RowSlice<T, LANES, PER>;
    constexpr int N = Slice::N;
    const float ct = scale_of(a);
    s.cut(base, lane, a.dim);
    if (marks) {
#pragma unroll
        for (int j = 0; j < (PER + 7) / 8; ++j) {
            const uint64_t mask = marks->of[lane][j];
            if (mask == 0) continue;
#pragma unroll
            for (int k = 0; k < 8 && j * 8 + k < PER; ++k) {
                uint32_t b = mask >> 8 * k & 0xff;
                if (b == 0) continue;
                if (base + Slice::COLUMNS > a.dim) b <<= Slice::skip(Slice::column(base, lane, j * 8 + k), a.dim);     // the last vector's elements are loaded further on in it
#pragma unroll
                for (int e = 0; e < N; ++e) if (b >> e & 1) s.x[j * 8 + k][e] = (T)-INFINITY;
            }
        }
    }
    s.forget();
    const float top = s.largest();
    s.forget();
    const Exponents f = exponents(top, ct);
    r.from = top;
    r.t = r.one = s.exponentials(f.scale, f.off) * f.back;
    if (a.alpha < 1.f && a.temperature != 1.f) {
        const Exponents f1 = exponents(top, LOG2E);
        s.forget();
        r.one = s.exponentials(f1.scale, f1.off) * f1.back;
    }
}
// of all the wavefronts of a row, in the first of them
template <int LANES>
__device__ __forceinline__ void join_waves(const DistillArgs& a, Sums& r, Sums* lds) {
    const bool two = a.alpha < 1.f && a.temperature != 1.f;
    const float ct = scale_of(a);
    r = r.over_wave(ct, two);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = r;
        __syncthreads();
        if (threadIdx.x >= 64) return;
        r = threadIdx.x < LANES / 64 ? lds[threadIdx.x] : NO_SUMS;
        r = r.over_wave(ct, two);
    }
}

// The gradient of a slice in the place of its logits, but for the named ids' and the target's.
template <class T, int LANES, int PER>
__device__ __forceinline__ void slice_grad(const DistillArgs& a, RowSlice<T, LANES, PER>& s, float g, const float* st) {
    const Exponents f = exponents(st[ST_REST], scale_of(a)), f1 = exponents(st[ST_REST], LOG2E);        // (their mends are in the coefficients)
    // (All lanes have the same.  Left to the compiler they are in vector registers, one wavefront a SIMD less for rows of 12,000 16-bit columns; us, none / these / all in scalar ones, loss and gradient
    // of 16,384 rows of 32,768 bf16 434 / 430 / 415, of 4000 of 24,000 91 / 87 / 88, of 131,072 487 / 467 / 464, of 8000 of 30,000 at temperature 2 218 / 224 / 233.)
    const float scale = scalar(f.scale), scale1 = scalar(f1.scale), coef = g * st[ST_COEF], coef1 = scalar(g * st[ST_COEF1]);
    const bool two = a.alpha < 1.f && a.temperature != 1.f;
    constexpr int N = RowSlice<T, LANES, PER>::N;
#pragma unroll
    for (int k = 0; k < PER; ++k) {                // (the choice inside: outside, every element would be converted before it)
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = coef * __builtin_amdgcn_exp2f(fmaf(s.at(k, e), scale, -f.off));
        if (two) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = fmaf(coef1, __builtin_amdgcn_exp2f(fmaf(s.at(k, e), scale1, -f1.off)), v[e]);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) s.x[k][e] = (T)v[e];
    }
}
// The gradients of the named ids and of the target in [base, end), after the slice is stored.  An id that is named several times is the first entry's.
template <class T, int LANES>
__device__ __forceinline__ void mend(const DistillArgs& a, float g, const float* st, const Entries& t, int y, float xy, int base, int end, int lane, T* out) {
    const float ct = scale_of(a), scale = a.alpha * a.temperature, hard = 1.f - a.alpha;
    const int entries = st[ST_KIND] == ROW_ENTRIES ? a.top : 0;
    const bool target = a.alpha < 1.f && y >= base && y < end;
    bool y_named = false;
    for (int k = lane; k < entries; k += LANES) {
        const int id = t.id[k];
        if (id < base || id >= end) continue;
        int times = 0;
        for (int j = 0; j < entries; j += 4) {
            const int4 q = *reinterpret_cast<const int4*>(t.id + j);
            times += (q.x == id) + (q.y == id) + (q.z == id) + (q.w == id);
        }
        float sum = t.z[k];
        bool first = true;
        if (times > 1) {
            sum = 0.f;
            for (int j = 0; j < entries; ++j)
                if (t.id[j] == id) { first &= j >= k; sum += t.z[j]; }
        }
        y_named |= id == y;
        if (!first) continue;
        const float d = t.x[k] - st[ST_ALL], q = exp2f(d * ct) * st[ST_INV], q1 = a.alpha < 1.f ? exp2f(d * LOG2E) * st[ST_INV1] : 0.f;
        out[id] = (T)(g * (scale * (st[ST_NAMED] * q - sum) + hard * (q1 - (id == y ? 1.f : 0.f))));
    }
    if (target) {                                  // (the same in all lanes of the row)
        if constexpr (LANES > 64) y_named = __syncthreads_or(y_named);
        else y_named = __any(y_named);
        if (!y_named && lane == 0) {
            const float rest = here(st[ST_REST]);
            const Exponents f = exponents(rest, ct);
            float v = g * st[ST_COEF] * __builtin_amdgcn_exp2f(fmaf(xy, f.scale, -f.off));
            if (a.temperature != 1.f) {
                const Exponents f1 = exponents(rest, LOG2E);
                v = fmaf(g * st[ST_COEF1], __builtin_amdgcn_exp2f(fmaf(xy, f1.scale, -f1.off)), v);
            }
            out[y] = (T)(v - g * hard);
        }
    }
}
template <class T, int LANES, int PER>
__device__ __forceinline__ void store_zeros(T* out, int base, int lane, int dim) {
    RowSlice<T, LANES, PER> s;
#pragma unroll
    for (int k = 0; k < PER; ++k) s.x[k] = typename RowSlice<T, LANES, PER>::V{};
    s.store(out, base, lane, dim, false);
}

constexpr int distill_threads(int lanes) { return lanes < 256 ? 256 : lanes; }

// Rows that LANES lanes hold: the loss, and the gradient too if it is wanted (grad), which may take the place of the logits: a row is read before any of it is written.  The row waits in
// registers while one wavefront works on its entries, so what counts is how many rows a compute unit holds: 80 registers and three rows of 64 KB, or four of 48, though some
// 30 bytes of a lane then go through memory (16,384 rows of 32,768 bf16, 4 to 8 wavefronts a SIMD: 475 / 475 / 412 / 471 / 549 us; at temperature 2 580 / 578 / 448 / 524 / 572).
template <class T, int LANES, int PER>
__global__ __launch_bounds__(distill_threads(LANES)) __attribute__((amdgpu_waves_per_eu(LANES > 512 ? 4 : LANES == 512 && PER == 6 ? 8 : 6))) void k_distill_row(DistillArgs a, bool stream, const float* __restrict__ grad_loss, int64_t grad_loss_stride, float* __restrict__ loss,
                                                                        float* __restrict__ stats, T* grad, int64_t grad_stride) {
    using Slice = RowSlice<T, LANES, PER>;
    constexpr int ROWS = distill_threads(LANES) / LANES;
    extern __shared__ __align__(16) float dynamic[];             // entries
    __shared__ Marks<LANES, PER> marks[ROWS];
    __shared__ Sums lds[distill_threads(LANES) / 64];
    __shared__ float row_stats[ROWS][STATS];
    const int lane = threadIdx.x % LANES, sub = LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / LANES) : threadIdx.x / LANES;
    const int64_t row = (int64_t)blockIdx.x * ROWS + sub;
    if (row >= a.n) return;                        // (all lanes of the row)
    const T* x = (const T*)a.x + row * a.stride;
    T* out = grad + (grad ? row * grad_stride : 0);
    Slice s;
    s.load(x, 0, lane, a.dim, stream);
    const float g = grad ? grad_loss[row * grad_loss_stride] : 0.f;
    int y;
    if (!row_target(a, row, &y)) {
        distill_left_out(row, lane, loss, stats);
        if (grad) store_zeros<T, LANES, PER>(out, 0, lane, a.dim);
        return;
    }
    const Entries t = entries_at(dynamic, sub, a.top);
    load_entries<T, LANES>(a, row, lane, x, t);
    const float xy = y >= 0 ? (float)x[y] : 0.f;
    const bool rest = a.lse && a.alpha > 0.f;
    if (rest) mark_named<T, LANES, PER>(a, row, 0, lane, marks[sub]);
    RowSums r{NO_SUMS, 0.f};
    add_slice<T, LANES, PER>(a, s, 0, lane, rest ? &marks[sub] : nullptr, r.rest);
    join_waves<LANES>(a, r.rest, lds);
    if (rest) r.twice = (float)marks[sub].twice;
    float* st = row_stats[sub];
    if constexpr (LANES <= 64) row_sync<LANES>();
    if (lane < 64) {
        distill_row(a, row, xy, r, t, loss, st);
        row_sync<64>();
        if (stats && lane < STATS) stats[row * STATS + lane] = st[lane];
    }
    if (!grad) return;
    row_sync<LANES>();
    if (st[ST_KIND] == ROW_OUT || g == 0.f) { store_zeros<T, LANES, PER>(out, 0, lane, a.dim); return; }
    s.forget();
    slice_grad<T, LANES, PER>(a, s, g, st);
    s.store(out, 0, lane, a.dim, stream);
    row_sync<LANES>();
    mend<T, LANES>(a, g, st, t, y, xy, 0, a.dim, lane, out);
}

// Sums of one slice of a longer row.
template <class T, int LANES, int PER>
__global__ __launch_bounds__(LOGIT_THREADS) void k_distill_slice(DistillArgs a, int slices, bool stream, RowSums* __restrict__ part) {
    using Slice = RowSlice<T, LANES, PER>;
    static_assert(LANES == LOGIT_THREADS);
    __shared__ Marks<LANES, PER> marks;
    __shared__ Sums lds[LOGIT_THREADS / 64];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x / slices;
    const int slice = blockIdx.x % slices, base = slice * Slice::COLUMNS;
    Slice s;
    s.load((const T*)a.x + row * a.stride, base, lane, a.dim, stream);
    if (a.target) {
        const int64_t y = load_id(a.target, a.target_type, row);
        if (y < 0 || y >= a.dim) return;
    }
    const bool rest = a.lse && a.alpha > 0.f;
    if (rest) mark_named<T, LANES, PER>(a, row, base, lane, marks);
    Sums r = NO_SUMS;
    add_slice<T, LANES, PER>(a, s, base, lane, rest ? &marks : nullptr, r);
    join_waves<LANES>(a, r, lds);
    if (lane == 0) part[row * slices + slice] = RowSums{r, rest ? (float)marks.twice : 0.f};
}

// The sums of a row's slices, by a wavefront.
__device__ __forceinline__ RowSums row_sums(const DistillArgs& a, const RowSums* __restrict__ part, int64_t row, int slices) {
    const float ct = scale_of(a);
    const bool two = a.alpha < 1.f && a.temperature != 1.f;
    RowSums r{NO_SUMS, 0.f};
    for (int k = threadIdx.x & 63; k < slices; k += 64) {
        const RowSums q = part[row * slices + k];
        r.rest.join(q.rest, ct, two);
        r.twice = fmaxf(r.twice, q.twice);
    }
    r.rest = r.rest.over_wave(ct, two);
    r.twice = __any(r.twice != 0.f) ? 1.f : 0.f;
    return r;
}

// The rows of several slices: a wavefront to a row.
template <class T>
__global__ __launch_bounds__(LOGIT_THREADS) void k_distill_join(DistillArgs a, int slices, const RowSums* __restrict__ part, float* __restrict__ loss, float* __restrict__ stats) {
    extern __shared__ __align__(16) float dynamic[];
    __shared__ float row_stats[LOGIT_THREADS / 64][STATS];
    const int lane = threadIdx.x & 63, sub = threadIdx.x / 64;
    const int64_t row = (int64_t)blockIdx.x * (LOGIT_THREADS / 64) + sub;
    if (row >= a.n) return;
    const T* x = (const T*)a.x + row * a.stride;
    const RowSums r = row_sums(a, part, row, slices);
    int y;
    if (!row_target(a, row, &y)) { distill_left_out(row, lane, loss, stats); return; }
    const Entries t = entries_at(dynamic, sub, a.top);
    load_entries<T, 64>(a, row, lane, x, t);
    const float xy = y >= 0 ? (float)x[y] : 0.f;
    row_sync<64>();
    distill_row(a, row, xy, r, t, loss, row_stats[sub]);
    row_sync<64>();
    if (lane < STATS) stats[row * STATS + lane] = row_stats[sub][lane];
}

// The gradient of a slice.  It may take the place of the logits: a slice is read, its entries among it, before any of it is written.
// PARTS: the row's sums of slices (`parts` of them) have not been joined; every workgroup does that for itself, which saves few rows a launch, and the first slice's stores the loss.  Not in place: a
// workgroup reads all of the row's entries, when others may have stored their slices.
template <class T, int LANES, int PER, bool PARTS>
__global__ __launch_bounds__(LOGIT_THREADS) void k_distill_bwd(DistillArgs a, int slices, bool stream, const RowSums* __restrict__ part, int parts, float* __restrict__ loss,
                                                               const float* __restrict__ grad_loss, int64_t grad_loss_stride, const float* __restrict__ stats, T* grad,
                                                               int64_t grad_stride) {
    using Slice = RowSlice<T, LANES, PER>;
    constexpr int ROWS = LOGIT_THREADS / LANES;
    static_assert(!PARTS || ROWS == 1);
    extern __shared__ __align__(16) float dynamic[];
    __shared__ float row_stats[PARTS ? STATS : 1];
    const int lane = threadIdx.x % LANES, sub = LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / LANES) : threadIdx.x / LANES;
    const int64_t row = (int64_t)(blockIdx.x / slices) * ROWS + sub;
    const int slice = blockIdx.x % slices, base = slice * Slice::COLUMNS;
    if (row >= a.n) return;
    const T* x = (const T*)a.x + row * a.stride;
    T* out = grad + row * grad_stride;
    Slice s;
    s.load(x, base, lane, a.dim, stream);
    const float g = grad_loss[row * grad_loss_stride];
    const int end = min(a.dim, base + Slice::COLUMNS);
    const Entries t = entries_at(dynamic, sub, a.top);
    const float* st = PARTS ? row_stats : stats + row * STATS;
    int y = -1;
    float xy = 0.f;
    if constexpr (PARTS) {
        if (!row_target(a, row, &y)) {
            if (slice == 0) distill_left_out(row, lane, loss, nullptr);
            store_zeros<T, LANES, PER>(out, base, lane, a.dim);
            return;
        }
        load_entries<T, LANES>(a, row, lane, x, t);
        if (y >= 0) xy = (float)x[y];
        __syncthreads();
        if (lane < 64) distill_row(a, row, xy, row_sums(a, part, row, parts), t, slice == 0 ? loss : nullptr, row_stats);
        __syncthreads();
        if (st[ST_KIND] == ROW_OUT || g == 0.f) { store_zeros<T, LANES, PER>(out, base, lane, a.dim); return; }
    } else {
        const float kind = st[ST_KIND];
        if (kind == ROW_OUT || g == 0.f) { store_zeros<T, LANES, PER>(out, base, lane, a.dim); return; }
        const double it = 1.0 / (double)a.temperature;
        for (int k = lane; kind == ROW_ENTRIES && k < a.top; k += LANES) {
            const int64_t i = row * a.top + k, id = load_id(a.ids, a.id_type, i);
            const bool here = id >= base && id < end;
            t.id[k] = here ? (int)id : -1;
            if (here) {
                t.z[k] = expf((float)exponent(load_value(a.z, a.z_type, i), st[ST_ZFROM], it)) * st[ST_ZINV];
                t.x[k] = (float)x[id];
            }
        }
        end_entries(t, lane, a.top);
        if (a.target && a.alpha < 1.f) {
            y = (int)load_id(a.target, a.target_type, row);
            if (y >= base && y < end) xy = (float)x[y];
        }
    }
    slice_grad<T, LANES, PER>(a, s, g, st);
    row_sync<LANES>();
    s.store(out, base, lane, a.dim, stream);
    row_sync<LANES>();
    mend<T, LANES>(a, g, st, t, y, xy, base, end, lane, out);
}

// Row-slices of one launch: what their sums take of the workspace, and what a launch can have of workgroups, is bounded; more rows go in several.
constexpr int64_t DISTILL_SLICES = 1 << 16;
constexpr size_t DISTILL_WORK = DISTILL_SLICES * (sizeof(RowSums) + STATS * sizeof(float));
size_t distill_work_bytes() { return DISTILL_WORK; }

// f(lanes of a slice, vectors of a lane), as constants, for the gradient of n rows of `vectors`.  Slices of 4 vectors a lane, or of 2 where those are fewer than four workgroups a
// compute unit.  us, 2 / 4: 32 rows of 131,072 bf16 (512 workgroups of 4) 6.9 / 7.4, 63 10.0 / 10.7, 96 13.6 / 13.4.  us, 8 / 4: 4096 rows of 131,072 bf16 363 / 353, 2000 182 / 170, 3000 of 50,021 155 / 115, 777 f16 38 / 31, 8000 of 30,000 bf16 165 / 161.
template <class F>
void by_slice(int64_t n, int64_t vectors, F f) {
    using std::integral_constant;
    if (vectors <= 64 * 2) f(integral_constant<int, 64>(), integral_constant<int, 2>());
    else if (vectors <= 64 * 8) f(integral_constant<int, 64>(), integral_constant<int, 8>());
    else if (n * cdiv(vectors, 256 * 4) < 1024) f(integral_constant<int, 256>(), integral_constant<int, 2>());
    else f(integral_constant<int, 256>(), integral_constant<int, 4>());
}
// f(vectors of a lane) for the sums of rows of more than 1024 vectors.  Slices of 8, or of 4 where the last one of 8 would be half empty, or more, among five at most, or of 2
// where there are few.  us, 2 / 8: 16 rows of 131,072 bf16 (128 slices of 8) 3.6 / 4.0, 32 4.4 / 4.2, 63 6.7 / 6.5, 96 8.7 / 8.0: the two are alike from 256 on.  us, 8 / 4: 4096 rows of 131,072 bf16 193 / 215, 8000 of 30,000 77 / 94, 4000 of 100,000 f32 228 / 240, but 3000 of 50,021 bf16 75 / 60.
template <class F>
void by_part(int64_t n, int64_t vectors, F f) {
    using std::integral_constant;
    const int64_t eights = cdiv(vectors, LOGIT_THREADS * 8);
    if (n * eights < 512) f(integral_constant<int, 2>());
    else if (eights <= 5 && cdiv(vectors, LOGIT_THREADS * 4) % 2 == 1) f(integral_constant<int, 4>());
    else f(integral_constant<int, 8>());
}
// the same for rows that one workgroup holds.  6 vectors a lane and not 8 where they are enough: idle lanes take registers from other rows, and with 512 lanes a fourth row fits a compute
// unit then.  us, 8 / 6: loss and gradient of 4000 rows of 10,000 bf16 62 / 53, of 12,000 65 / 56, of 17,000 108 / 91, of 24,000 113 / 99, of 10,000 f32 83 / 75 (with 512 lanes at three rows a
// compute unit 96, 106 and 83, the last three; four rows with 256 lanes 55 and 60, the first two).
constexpr int64_t ROW_MOST = 1024 * 16;
template <class F>
void by_row(int64_t vectors, F f) {
    using std::integral_constant;
    if (vectors <= 64 * 2) f(integral_constant<int, 64>(), integral_constant<int, 2>());
    else if (vectors <= 64 * 8) f(integral_constant<int, 64>(), integral_constant<int, 8>());
    else if (vectors <= 256 * 4) f(integral_constant<int, 256>(), integral_constant<int, 4>());
    else if (vectors <= 256 * 6) f(integral_constant<int, 256>(), integral_constant<int, 6>());
    else if (vectors <= 256 * 8) f(integral_constant<int, 256>(), integral_constant<int, 8>());
    else if (vectors <= 512 * 6) f(integral_constant<int, 512>(), integral_constant<int, 6>());
    else if (vectors <= 512 * 8) f(integral_constant<int, 512>(), integral_constant<int, 8>());
    else if (vectors <= 1024 * 8) f(integral_constant<int, 1024>(), integral_constant<int, 8>());
    else f(integral_constant<int, 1024>(), integral_constant<int, 16>());
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

// Rows below which the gradient's kernel joins the slices, and no workgroup of 1024 takes a row.  us a call, joined by it / by a kernel of its own / whole rows: temperature 2, 131,072 bf16: one row 14.4 / 17.4,
// 32 14.2 / 17.8, 63 18.5 / 21.5, 128 27.6 / 31.1, 256 47.3 / 47.8; temperature 1: 32 13.5 / 15.9 / 20.4, 64 17.3 / 21.5 / 22.6, 96 20.7 / 24.6 / 25.3, 128 23.6 / 27.5 / 27.4, 256 42.1 / 42.6 / 36.8: the gradient's
// kernel is ahead up to some 200 rows.
constexpr int64_t DISTILL_FEW = 64;
// Whether a workgroup takes a whole row, in one launch, or rows are cut into slices.  Loss and gradient: rows of up to 4096 vectors; larger ones, of which a compute unit holds two or
// one, only where they leave few lanes idle and have one exponential an element (nothing else runs while a workgroup works).  us, whole rows / slices, bf16: 16,384 rows of 32,768 430 / 564,
// 4000 of 20,000 95 / 116; one exponential: 4000 of 131,072 476 / 504, 300 of 65,536 30 / 33, 4000 of 60,000 271 / 253 (f32, 2000 of 30,000, 114 / 129), of 50,021 335 / 268;
// two exponentials: 4000 of 131,072 582 / 533, of 65,536 314 / 276.  The loss alone: 16,000 rows of 16,000 bf16 130 / 116, of 30,000 230 / 178, but 256 of 30,000
// 10.7 / 12.8, 1024 17.0 / 20.2, 2048 30.9 / 32.7, 4000 52.6 / 54.0, and of 16,000 12.1 / 15.2 (1024), 29.3 / 36.0 (4000): the two meet beyond 4000 rows.
static bool in_one_workgroup(const DistillCall& c, int64_t vectors) {
    if (!c.bwd) return vectors <= 256 * 4 || (vectors <= 512 * 8 && c.a.n <= 1024);
    if (vectors <= 512 * 8) return true;
    const bool two = c.a.alpha < 1.f && c.a.temperature != 1.f;
    return !two && c.a.n >= DISTILL_FEW && vectors <= ROW_MOST && vectors * 8 >= (vectors <= ROW_MOST / 2 ? ROW_MOST / 2 : ROW_MOST) * 7;
}

template <class T>
int distill_run(const DistillCall& c) {
    constexpr int N = VECTOR<T>;
    const DistillArgs& a = c.a;
    const hipStream_t st = c.d->stream;
    const int64_t vectors = cdiv(a.dim, N);
    const size_t entry_bytes = (size_t)entries_room(a.top) * 12;
    // Logits that the memory-side cache does not hold until the next pass (256 MB, the gradient among them) stay out of its way.  us: 8192 rows of 131,072 bf16 (2.1 GB), loss
    // 357 / 319; 4096 such rows, the loss before its gradient 218 / 183; but 777 of 50,021 f16 (78 MB), loss and then gradient 74 / 81.
    const bool stream = a.n * a.dim * (int64_t)sizeof(T) > (int64_t)128 << 20;
    if (c.fwd && in_one_workgroup(c, vectors)) {
        by_row(vectors, [&](auto l, auto p) {
            constexpr int LANES = decltype(l)::value, PER = decltype(p)::value, THREADS = distill_threads(LANES), ROWS = THREADS / LANES;
            const int64_t most = LAUNCH_THREADS / LANES;
            for (int64_t at = 0; at < a.n; at += most) {
                const DistillArgs b = rows_of(a, at, std::min(most, a.n - at), sizeof(T));
                k_distill_row<T, LANES, PER><<<(unsigned)cdiv(b.n, ROWS), THREADS, ROWS * entry_bytes, st>>>(
                    b, stream, c.grad_loss + at * c.grad_loss_stride, c.grad_loss_stride, c.loss + at, c.stats ? c.stats + at * STATS : nullptr,
                    c.grad ? (T*)c.grad + at * c.grad_stride : nullptr, c.grad_stride);
            }
        });
        FC_HIP(hipGetLastError());
        return FC_OK;
    }
    if (c.fwd) FC_TRY(dense_work(c.d, DISTILL_WORK));
    RowSums* part = reinterpret_cast<RowSums*>(c.d->work);
    float* work_stats = reinterpret_cast<float*>(c.d->work + DISTILL_SLICES * sizeof(RowSums));
    const bool joins = c.fwd && c.bwd && !c.stats && a.n < DISTILL_FEW && c.grad != a.x;      // the gradient's kernel joins the slices
    int parts = 1;                                 // slices of a row's sums
    if (c.fwd) by_part(a.n, vectors, [&](auto p) { parts = (int)cdiv(vectors, LOGIT_THREADS * decltype(p)::value); });
    // rows of a launch: as many as the workspace has slices for, or as a launch has workgroups for (the smallest slices have 128 vectors)
    const int64_t most = c.fwd ? DISTILL_SLICES / parts : LAUNCH_THREADS / LOGIT_THREADS / cdiv(vectors, 128);
    for (int64_t at = 0; at < a.n; at += most) {
        const int64_t n = std::min(most, a.n - at);
        const DistillArgs b = rows_of(a, at, n, sizeof(T));
        float* stats = c.stats ? c.stats + at * STATS : work_stats;
        if (c.fwd) {
            by_part(a.n, vectors, [&](auto p) {
                constexpr int PER = decltype(p)::value;
                k_distill_slice<T, LOGIT_THREADS, PER><<<(unsigned)(n * parts), LOGIT_THREADS, 0, st>>>(b, parts, stream, part);
            });
            if (!joins)
                k_distill_join<T><<<(unsigned)cdiv(n, LOGIT_THREADS / 64), LOGIT_THREADS, LOGIT_THREADS / 64 * entry_bytes, st>>>(b, parts, part, c.loss + at, stats);
        }
        if (!c.bwd) continue;
        by_slice(a.n, vectors, [&](auto l, auto p) {
            constexpr int LANES = decltype(l)::value, PER = decltype(p)::value, ROWS = LOGIT_THREADS / LANES;
            auto backward = [&](auto joining) {
                const int64_t slices = cdiv(vectors, LANES * PER);
                k_distill_bwd<T, LANES, PER, decltype(joining)::value><<<(unsigned)(cdiv(n, ROWS) * slices), LOGIT_THREADS, ROWS * entry_bytes, st>>>(
                    b, (int)slices, stream, part, parts, c.loss ? c.loss + at : nullptr, c.grad_loss + at * c.grad_loss_stride, c.grad_loss_stride, stats,
                    (T*)c.grad + at * c.grad_stride, c.grad_stride);
            };
            if constexpr (LANES == LOGIT_THREADS)
                if (joins) { backward(std::true_type()); return; }
            backward(std::false_type());
        });
    }
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
