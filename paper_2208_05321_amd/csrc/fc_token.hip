// Token embedding: rows of a table in the model's type, scaled, and the table's gradient by sorted tokens.
//
//   forward   out[i, :] = T(scale * table[ids[i], :])
//   backward  grad[v, :] (+)= scale * sum over the tokens i with ids[i] == v of grad_out[i, :]
//
// Backward: the tokens are put in order by id with the sort of the bags' backward pass (stable, so that an id's tokens keep their
// order) and every row of the gradient is written once, by the lanes that add its tokens up; without accumulation a row without
// tokens gets its zeros in the same pass.  Popular ids are what a sum by rows has to be protected from: the sorted tokens are cut
// into chunks of 64, and a chunk that lies inside one id's run is added up beforehand, by lanes of its own, as are 64 such chunks
// in a row.  A row then adds at most 126 tokens, 126 chunks and n / 4096 stretches, whatever the ids.  All sums are in 32 bits and in
// an order that depends on the ids alone: results are reproducible.
#include "dense_device.h"

#include <algorithm>

namespace fc {

constexpr int TOK_THREADS = 256;
constexpr int TOK_CHUNK = 64;                     // sorted tokens to a chunk, and chunks to a stretch
constexpr int TOK_STRETCH = TOK_CHUNK * TOK_CHUNK;

// ---- forward ----
template <int ROWS, class S, class D, class I>
__global__ __launch_bounds__(TOK_THREADS) void k_token_fwd(const S* __restrict__ table, int64_t table_stride, int rows, int dim, int lpr_shift,
                                                           const I* __restrict__ ids, int64_t n, float scale, D* __restrict__ out,
                                                           int64_t out_stride, uint32_t* flags) {
    constexpr int N = VECTOR<S>;
    const int lpr = 1 << lpr_shift, lane = threadIdx.x & (lpr - 1);
    const int64_t first = (((int64_t)blockIdx.x * TOK_THREADS + threadIdx.x) >> lpr_shift) * ROWS;
    const S* row[ROWS];
    bool bad = false;
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const I id = ids[min(first + k, n - 1)];
        const bool ok = id >= 0 && id < (I)rows;
        bad |= !ok;
        row[k] = ok ? table + (size_t)id * table_stride : nullptr;
    }
    if (bad && lane == 0 && first < n) atomicOr(flags, EF_ID_RANGE);
    for (int col = lane * N; col < dim; col += lpr * N) {
        float v[ROWS][N];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            if (row[k]) load_as_float(v[k], row[k] + col, dim - col);
            else
#pragma unroll
                for (int e = 0; e < N; ++e) v[k][e] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            if (first + k >= n) break;
            // (a row of an id outside stays zero even where the scale is infinite)
#pragma unroll
            for (int e = 0; e < N; ++e) v[k][e] = row[k] ? v[k][e] * scale : 0.f;
            store_from_float(out + (first + k) * out_stride + col, v[k], dim - col);
        }
    }
}

// ---- backward ----
// Sort keys: the id, or `rows` for the padding id and for ids outside.  first: one word per table row, "no token" to begin with.
template <class I>
__global__ __launch_bounds__(TOK_THREADS) void k_token_keys(const I* __restrict__ ids, int64_t n, int rows, int64_t padding_id, int32_t* __restrict__ keys,
                                                            int32_t* __restrict__ first, uint32_t* flags) {
    const int64_t i = (int64_t)blockIdx.x * TOK_THREADS + threadIdx.x;
    bool bad = false;
    if (i < n) {
        const I id = ids[i];
        const bool ok = id >= 0 && id < (I)rows;
        bad = !ok && (int64_t)id != padding_id;
        keys[i] = ok && (int64_t)id != padding_id ? (int)id : rows;
    }
    if (first && i < rows) first[i] = -1;
    if (bad) atomicOr(flags, EF_ID_RANGE);
}

// acc += rows vals[a .. b) of grad_out, columns from `col`, in order
template <int N, class S>
__device__ __forceinline__ void add_tokens(float (&acc)[N], const S* __restrict__ grad_out, int64_t stride, const int32_t* __restrict__ vals, int a, int b,
                                           int col, int dim) {
    constexpr int AT_ONCE = 8;
    for (; a + AT_ONCE <= b; a += AT_ONCE) {
        float v[AT_ONCE][N];
        int at[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) at[k] = vals[a + k];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) load_as_float(v[k], grad_out + (size_t)at[k] * stride + col, dim - col);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += v[k][e];
    }
    for (; a < b; ++a) {
        float v[N];
        load_as_float(v, grad_out + (size_t)vals[a] * stride + col, dim - col);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += v[e];
    }
}
// the same for partial rows [a .. b), which are `dim` floats apart
template <int N>
__device__ __forceinline__ void add_parts(float (&acc)[N], const float* __restrict__ part, int a, int b, int col, int dim) {
#pragma unroll 4
    for (; a < b; ++a) {
        float v[N];
        load_as_float(v, part + (size_t)a * dim + col, dim - col);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += v[e];
    }
}

// Chunks inside one id's run are added up; first[id] = where its run begins.
template <class S>
__global__ __launch_bounds__(TOK_THREADS) void k_token_chunks(const S* __restrict__ grad_out, int64_t stride, const int32_t* __restrict__ keys,
                                                              const int32_t* __restrict__ vals, int n, int rows, int dim, int lpr_shift,
                                                              float* __restrict__ part, int32_t* __restrict__ first) {
    constexpr int N = VECTOR<S>;
    const int lpr = 1 << lpr_shift, lane = threadIdx.x & (lpr - 1);
    const int64_t chunk = ((int64_t)blockIdx.x * TOK_THREADS + threadIdx.x) >> lpr_shift;
    const int64_t a = chunk * TOK_CHUNK;
    if (a >= n) return;
    if (first)
        for (int j = lane; j < TOK_CHUNK && a + j < n; j += lpr) {
            const int key = keys[a + j];
            if (key < rows && (a + j == 0 || keys[a + j - 1] != key)) first[key] = (int)(a + j);
        }
    if (a + TOK_CHUNK > n || keys[a] == rows || keys[a] != keys[a + TOK_CHUNK - 1]) return;
    for (int col = lane * N; col < dim; col += lpr * N) {
        float acc[N] = {};
        add_tokens(acc, grad_out, stride, vals, (int)a, (int)a + TOK_CHUNK, col, dim);
        store_from_float(part + chunk * dim + col, acc, dim - col);
    }
}

// Stretches inside one id's run: the chunks' sums added up.
__global__ __launch_bounds__(TOK_THREADS) void k_token_stretches(const int32_t* __restrict__ keys, int n, int rows, int dim, int lpr_shift,
                                                                 const float* __restrict__ part, float* __restrict__ far_part) {
    constexpr int N = 4;
    const int lpr = 1 << lpr_shift, lane = threadIdx.x & (lpr - 1);
    const int64_t s = ((int64_t)blockIdx.x * TOK_THREADS + threadIdx.x) >> lpr_shift, a = s * TOK_STRETCH;
    if (a + TOK_STRETCH > n || keys[a] == rows || keys[a] != keys[a + TOK_STRETCH - 1]) return;
    for (int col = lane * N; col < dim; col += lpr * N) {
        float acc[N] = {};
        add_parts(acc, part, (int)s * TOK_CHUNK, ((int)s + 1) * TOK_CHUNK, col, dim);
        store_from_float(far_part + s * dim + col, acc, dim - col);
    }
}

// end of the run of `key` that holds position i
__device__ __forceinline__ int run_end(const int32_t* __restrict__ keys, int n, int i, int key) {
    int64_t step = 1;
    while (i + step < n && keys[i + step] == key) step <<= 1;
    int lo = (int)(i + step / 2), hi = (int)min((int64_t)n, i + step);       // keys[lo] is in, hi is out
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] == key) lo = mid; else hi = mid;
    }
    return hi;
}

template <int N, class S>
__device__ __forceinline__ void add_run(float (&acc)[N], const S* __restrict__ grad_out, int64_t stride, const int32_t* __restrict__ vals, int a, int b,
                                        const float* __restrict__ part, const float* __restrict__ far_part, int col, int dim) {
    int c = (a + TOK_CHUNK - 1) / TOK_CHUNK;
    const int c1 = b / TOK_CHUNK;
    if (c >= c1) { add_tokens(acc, grad_out, stride, vals, a, b, col, dim); return; }
    add_tokens(acc, grad_out, stride, vals, a, c * TOK_CHUNK, col, dim);
    int s = (c + TOK_CHUNK - 1) / TOK_CHUNK;
    const int s1 = c1 / TOK_CHUNK;
    if (s < s1) {
        add_parts(acc, part, c, s * TOK_CHUNK, col, dim);
        add_parts(acc, far_part, s, s1, col, dim);
        c = s1 * TOK_CHUNK;
    }
    add_parts(acc, part, c, c1, col, dim);
    add_tokens(acc, grad_out, stride, vals, c1 * TOK_CHUNK, b, col, dim);
}

// ADD: the lanes of a row-group look at PER sorted positions and take the rows whose runs begin there; else at PER rows of the gradient.
template <bool ADD, int PER, class S, class G>
__global__ __launch_bounds__(TOK_THREADS) void k_token_rows(const S* __restrict__ grad_out, int64_t stride, const int32_t* __restrict__ keys,
                                                            const int32_t* __restrict__ vals, int n, int rows, int dim, int lpr_shift, float scale,
                                                            const float* __restrict__ part, const float* __restrict__ far_part,
                                                            const int32_t* __restrict__ first, G* __restrict__ grad, int64_t grad_stride) {
    constexpr int N = VECTOR<S>;
    const int lpr = 1 << lpr_shift, lane = threadIdx.x & (lpr - 1);
    const int64_t at = (((int64_t)blockIdx.x * TOK_THREADS + threadIdx.x) >> lpr_shift) * PER;
    const int64_t end = ADD ? n : rows;
    for (int k = 0; k < PER && at + k < end; ++k) {
        int row, a;
        if (ADD) {
            a = (int)(at + k);
            row = keys[a];
            if (row == rows || (a > 0 && keys[a - 1] == row)) continue;
        } else {
            row = (int)(at + k);
            a = first[row];
        }
        const int b = a < 0 ? a : run_end(keys, n, a, row);
        G* const out = grad + (size_t)row * grad_stride;
        for (int col = lane * N; col < dim; col += lpr * N) {
            float acc[N] = {};
            if (a < b) add_run(acc, grad_out, stride, vals, a, b, part, far_part, col, dim);
            float old[N] = {};
            if (ADD) load_as_float(old, out + col, dim - col);
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] = ADD ? fmaf(acc[e], scale, old[e]) : a < b ? acc[e] * scale : 0.f;
            store_from_float(out + col, acc, dim - col);
        }
    }
}

template <class G>
__global__ __launch_bounds__(TOK_THREADS) void k_token_no_rows(G* __restrict__ grad, int64_t stride, int64_t rows, int dim) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int c = threadIdx.x; c < dim; c += TOK_THREADS) grad[r * stride + c] = (G)0.f;
}

struct TokenWork { size_t keys, first, part, far_part, bytes; };
static TokenWork token_work(int64_t n, int64_t rows, int64_t dim) {
    TokenWork w;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t p = at; at += (bytes + 255) & ~(size_t)255; return p; };
    w.keys = take((size_t)n * 4);
    w.first = take((size_t)rows * 4);
    w.part = take((size_t)(n / TOK_CHUNK) * dim * 4);
    w.far_part = take((size_t)(n / TOK_STRETCH) * dim * 4);
    w.bytes = at;
    return w;
}
size_t token_work_bytes(int64_t n, int64_t rows, int64_t dim) { return token_work(n, rows, dim).bytes; }

static int shift_for(int64_t dim, int per_lane) {
    return __builtin_ctz(pow2_from(cdiv(dim, per_lane), TOK_THREADS));
}

template <class S, class G>
static int token_bwd(fc_dense* d, const S* grad_out, int64_t stride, const int32_t* keys, int64_t n, int64_t rows, int dim, float scale, const TokenWork& w,
                     G* grad, int64_t grad_stride, bool add) {
    const hipStream_t st = d->stream;
    int bits = 1;
    while (((int64_t)1 << bits) <= rows) ++bits;                 // keys lie in [0, rows]
    SortJob j;
    j.src = SORT_SRC_SLOTS; j.keys_in = keys; j.n = (int)n; j.num_bags = (int)n; j.one_per_bag = true; j.limit = (int)rows; j.bits = bits;
    const int32_t *ks, *vs;
    FC_TRY(sort_in(j, d->sort, st, &ks, &vs));
    float* part = reinterpret_cast<float*>(d->work + w.part);
    float* far_part = reinterpret_cast<float*>(d->work + w.far_part);
    int32_t* first = add ? nullptr : reinterpret_cast<int32_t*>(d->work + w.first);
    const int sh = shift_for(dim, VECTOR<S>);
    const int64_t chunks = cdiv(n, TOK_CHUNK);
    k_token_chunks<<<(unsigned)cdiv(chunks << sh, TOK_THREADS), TOK_THREADS, 0, st>>>(grad_out, stride, ks, vs, (int)n, (int)rows, dim, sh, part, first);
    if (n >= TOK_STRETCH) {
        const int s4 = shift_for(dim, 4);
        k_token_stretches<<<(unsigned)cdiv((n / TOK_STRETCH) << s4, TOK_THREADS), TOK_THREADS, 0, st>>>(ks, (int)n, (int)rows, dim, s4, part, far_part);
    }
    constexpr int PER = 4;
    const unsigned blocks = (unsigned)cdiv(cdiv(add ? n : rows, PER) << sh, TOK_THREADS);
    if (add) k_token_rows<true, PER><<<blocks, TOK_THREADS, 0, st>>>(grad_out, stride, ks, vs, (int)n, (int)rows, dim, sh, scale, part, far_part, first, grad, grad_stride);
    else k_token_rows<false, PER><<<blocks, TOK_THREADS, 0, st>>>(grad_out, stride, ks, vs, (int)n, (int)rows, dim, sh, scale, part, far_part, first, grad, grad_stride);
    FC_HIP(hipGetLastError());
    return FC_OK;
}

}  // namespace fc

using namespace fc;

extern "C" {

int token_embed_fwd(fc_dense* d, const void* table_dev, int32_t table_type, int64_t table_stride, int64_t num_rows, int32_t dim, const void* ids_dev,
                    int32_t id_type, int64_t n, float scale, void* out_dev, int32_t out_type, int64_t out_stride) {
    if (!d || n < 0 || n >= DENSE_LIMIT || num_rows <= 0 || num_rows >= DENSE_LIMIT || dim <= 0 || dim > DENSE_MAX_DIM || table_stride < dim ||
        out_stride < dim || !is_float_type(table_type) || !is_float_type(out_type) || (id_type != FC_TYPE_I32 && id_type != FC_TYPE_I64) ||
        (n > 0 && (!table_dev || !ids_dev || !out_dev)))
        return FC_ERR_INVALID_ARG;
    if (n == 0) return FC_OK;
    FC_HIP(hipSetDevice(d->device));
    return with_type(table_type, [&](auto s) -> int {
        return with_type(out_type, [&](auto o) -> int {
            using S = decltype(s);
            using D = decltype(o);
            const int sh = shift_for(dim, VECTOR<S>);
            auto run = [&](auto id) {
                using I = decltype(id);
                k_token_fwd<1><<<(unsigned)cdiv(n << sh, TOK_THREADS), TOK_THREADS, 0, d->stream>>>(
                    (const S*)table_dev, table_stride, (int)num_rows, dim, sh, (const I*)ids_dev, n, scale, (D*)out_dev, out_stride, d->flags);
            };
            if (id_type == FC_TYPE_I32) run(int32_t()); else run(int64_t());
            FC_HIP(hipGetLastError());
            return FC_OK;
        });
    });
}

int token_embed_bwd(fc_dense* d, const void* grad_out_dev, int32_t grad_out_type, int64_t grad_out_stride, const void* ids_dev, int32_t id_type, int64_t n,
                    int64_t num_rows, int32_t dim, float scale, int64_t padding_id, void* grad_table_dev, int32_t grad_table_type,
                    int64_t grad_table_stride, int32_t accumulate) {
    if (!d || n < 0 || n >= DENSE_LIMIT || num_rows <= 0 || num_rows >= DENSE_LIMIT || dim <= 0 || dim > DENSE_MAX_DIM || grad_out_stride < dim ||
        grad_table_stride < dim || !is_float_type(grad_out_type) || (grad_table_type != FC_TYPE_F32 && grad_table_type != grad_out_type) ||
        (id_type != FC_TYPE_I32 && id_type != FC_TYPE_I64) || !grad_table_dev || (n > 0 && (!grad_out_dev || !ids_dev)))
        return FC_ERR_INVALID_ARG;
    if (n == 0 && accumulate) return FC_OK;
    FC_HIP(hipSetDevice(d->device));
    const hipStream_t st = d->stream;
    const TokenWork w = token_work(n, accumulate ? 0 : num_rows, dim);
    if (n > 0) {
        FC_TRY(ensure_sort(d->sort, n));
        FC_TRY(dense_work(d, w.bytes));
        int32_t* keys = reinterpret_cast<int32_t*>(d->work + w.keys);
        int32_t* first = accumulate ? nullptr : reinterpret_cast<int32_t*>(d->work + w.first);
        const unsigned blocks = (unsigned)cdiv(std::max<int64_t>(n, accumulate ? 0 : num_rows), TOK_THREADS);
        if (id_type == FC_TYPE_I32)
            k_token_keys<<<blocks, TOK_THREADS, 0, st>>>((const int32_t*)ids_dev, n, (int)num_rows, padding_id, keys, first, d->flags);
        else k_token_keys<<<blocks, TOK_THREADS, 0, st>>>((const int64_t*)ids_dev, n, (int)num_rows, padding_id, keys, first, d->flags);
    }
    return with_type(grad_out_type, [&](auto s) -> int {
        using S = decltype(s);
        auto go = [&](auto* grad) -> int {
            if (n == 0) {
                k_token_no_rows<<<(unsigned)std::min<int64_t>(num_rows, 65536), TOK_THREADS, 0, st>>>(grad, grad_table_stride, num_rows, dim);
                FC_HIP(hipGetLastError());
                return FC_OK;
            }
            return token_bwd(d, (const S*)grad_out_dev, grad_out_stride, reinterpret_cast<const int32_t*>(d->work + w.keys), n, num_rows, dim, scale, w,
                             grad, grad_table_stride, accumulate != 0);
        };
        return grad_table_type == FC_TYPE_F32 ? go((float*)grad_table_dev) : go((S*)grad_table_dev);
    });
}

}  // extern "C"
