// Token embedding: rows of a table in the model's type, scaled, and the table's gradient by sorted tokens.
//
//   forward   out[i, :] = T(scale * table[ids[i], :])
//   backward  grad[v, :] (+)= scale * sum over the tokens i with ids[i] == v of grad_out[i, :]
//
// Backward: the tokens are put in order by id with the sort of the bags' backward pass (stable, so that an id's tokens keep their
// order) and every row of the gradient is written once, by the lanes that add its tokens up; without accumulation a row without
// tokens gets its zeros in the same pass.  Popular ids are what a sum by rows has to be protected from: the sorted tokens are cut
// into chunks of 16, and a chunk that lies inside one id's run is added up beforehand, by lanes of its own, as are 16 such chunks
// in a row (a stretch) and, from 65,536 tokens on, 16 stretches (a mile).  A row then adds at most 30 tokens, 30 chunks, 30 stretches and n / 4096 miles,
// whatever the ids; with fewer tokens there are no miles, and it adds up to n / 256 stretches, 255 at most.  All sums are in 32 bits and in an order that depends on the ids alone: results are reproducible.
// HBM bounds the large calls (the zeros of the dense gradient alone are 142 us of the 226 that one of 131,072 rows of 2048 columns takes with 16 k tokens),
// the chain sort - chunks - rows the others: 426 k tokens of 128 columns added to 1 M rows 98 us, 32 of them the sort and 28 the chunks.
// (With chunks of 64 a popular row's 126 tokens, one after the other, were the kernel's duration: dense gradient of 131,072 rows of 2048
// columns, 16,384 tokens, 330 us.)
#include "dense_device.h"

#include <algorithm>
#include <type_traits>

namespace fc {

constexpr int TOK_THREADS = 256;
constexpr int TOK_CHUNK = 16;                     // sorted tokens to a chunk, chunks to a stretch, stretches to a mile
constexpr int TOK_STRETCH = TOK_CHUNK * TOK_CHUNK, TOK_MILE = TOK_CHUNK * TOK_STRETCH;
constexpr int64_t TOK_MILES_FROM = 16 * TOK_MILE;  // tokens from which on miles are added up: fewer cost a row less than the launch
constexpr int64_t TOK_MOST = (int64_t)1 << 36;    // tokens x columns of a gradient: the lanes of its runs fit a launch
constexpr int TOK_BLOCK = 64;                     // sorted tokens whose run heads are one word

// ---- columns ----
// A row is walked in vectors of N columns, a lane each.  The last one ends with the row: where the width is no multiple of N it overlaps the one
// before it, and both lanes work out, and store, the same values in the columns that they share.  (With a partial vector handled wherever one is loaded or
// stored the backward pass's kernels grew to 1200 branches and waited for their own instructions: dense gradient of 131,072 rows of 2048 columns 380
// us; with the columns left over done after the others every row took its chain of loads twice: 1.8 M rows of 55, 436 k tokens 191.)  Rows
// narrower than a vector have kernels with N = 1.
// Cols: first columns of the U vectors that a lane takes of a row, -1 where it has none.
template <int U> struct Cols { int at[U]; };
// Workgroups that share a row's columns are neighbours; each has `per_tile` vectors.
struct Tiles { int dim, lpr_shift, per_tile, tiles; };
template <int U, int N>
__device__ __forceinline__ Cols<U> my_cols(const Tiles& q, int tile) {
    const int lane = threadIdx.x & ((1 << q.lpr_shift) - 1), end = min((q.dim + N - 1) / N, (tile + 1) * q.per_tile);
    Cols<U> c;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = tile * q.per_tile + (u << q.lpr_shift) + lane;
        c.at[u] = v < end ? min(v * N, q.dim - N) : -1;
    }
    return c;
}
struct Tile { unsigned block; int tile; };
__device__ __forceinline__ Tile my_tile(const Tiles& q) {
    const unsigned b = blockIdx.x / (unsigned)q.tiles;
    return Tile{b, (int)(blockIdx.x - b * (unsigned)q.tiles)};
}
static Tiles tiles_of(int dim, int per_lane, int vectors) {
    const int nv = (int)cdiv(dim, per_lane), sh = __builtin_ctz(pow2_from(nv, 64));
    Tiles q{dim, sh, 0, (int)cdiv(nv, vectors << sh)};
    q.per_tile = (int)cdiv(nv, q.tiles);
    // two vectors that overlap belong to one wavefront: it reads what it adds to before it stores anything
    while (q.tiles > 1 && dim % per_lane && (nv - 1) % q.per_tile == 0) { --q.per_tile; q.tiles = (int)cdiv(nv, q.per_tile); }
    return q;
}

// ---- forward ----
// out = T(scale * row): a row-group, or a workgroup, reads its row's id and copies; nothing is shared, so a lane's loads all leave at once.  HBM bounds it:
// 8192 rows of 4096 16-bit columns 16 to 17 us (89 MB, 5.3 TB/s, a large copy's rate), 426 k of 64 f32 to bf16 16 to 18 us; one row 1.7 us, the launch.
template <int ROWS, int N, class S, class D, class I>
__global__ __launch_bounds__(TOK_THREADS) void k_token_fwd(const S* __restrict__ table, int64_t table_stride, int rows, int dim, int lpr_shift,
                                                           const I* __restrict__ ids, int64_t n, float scale, D* __restrict__ out,
                                                           int64_t out_stride, uint32_t* flags) {
    const int lpr = 1 << lpr_shift, lane = threadIdx.x & (lpr - 1), vectors = (dim + N - 1) / N;
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
    for (int c = lane; c < vectors; c += lpr) {
        const int col = min(c * N, dim - N);
        float v[ROWS][N];
#pragma unroll
        for (int k = 0; k < ROWS; ++k)
            if (row[k]) load_vector(v[k], row[k] + col);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            if (first + k >= n) break;
            // (a row of an id outside stays zero even where the scale is infinite)
#pragma unroll
            for (int e = 0; e < N; ++e) v[k][e] = row[k] ? v[k][e] * scale : 0.f;
            store_vector(out + (first + k) * out_stride + col, v[k]);
        }
    }
}

// ---- backward ----
// Where an id's tokens begin and end among the sorted ones; begin < 0: it has none.
struct TokenRun { int begin, end; };

// Sort keys: the id, or `rows` for the padding id and for ids outside.  (-1 says that there is no padding id: as an id it is one outside, as in the
// forward pass.)  runs: one per table row, without tokens to begin with.
template <class I>
__device__ __forceinline__ int token_key(I id, int rows, int64_t padding_id, bool& bad) {
    const bool ok = id >= 0 && id < (I)rows, pad = padding_id != -1 && (int64_t)id == padding_id;
    bad |= !ok && !pad;
    return ok && !pad ? (int)id : rows;
}
template <class I>
__global__ __launch_bounds__(TOK_THREADS) void k_token_keys(const I* __restrict__ ids, int64_t n, int rows, int64_t padding_id, int32_t* __restrict__ keys,
                                                            TokenRun* __restrict__ runs, uint32_t* flags) {
    const int64_t i = (int64_t)blockIdx.x * TOK_THREADS + threadIdx.x;
    bool bad = false;
    if (i < n) keys[i] = token_key(ids[i], rows, padding_id, bad);
    if (runs && i < rows) runs[i] = TokenRun{-1, -1};
    if (bad) atomicOr(flags, EF_ID_RANGE);
}

// Rows that a lane has on their way together: 32 sums' worth.  More of them, or two vectors of eight columns to a lane, cost wavefronts.
// us a call, 8 rows and two vectors / 4 and one: 37 k tokens added to 137 k rows of 2048 16-bit columns 114 / 101, 426 k to 1 M of 128 107.5 / 97.
template <int U, int N> constexpr int token_loads = 32 / (U * N) < 8 ? 32 / (U * N) : 8;

// acc += the rows at(a) .. at(b - 1) of src, in order.  AT rows' loads are on their way together; the last ones that do not make AT go in halves
// of it, with the last row read again in the place of rows beyond it, and not counted.
template <int AT, int U, int N, class S, class F>
__device__ __forceinline__ void add_rows(float (&acc)[U][N], const S* __restrict__ src, int64_t stride, F at, int a, int b, const Cols<U>& c) {
    auto batch = [&](auto size, bool whole) {
        constexpr int B = decltype(size)::value;
        int p[B];
#pragma unroll
        for (int k = 0; k < B; ++k) p[k] = at(whole ? a + k : min(a + k, b - 1));
        float v[B][U][N];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c.at[u] >= 0)
#pragma unroll
                for (int k = 0; k < B; ++k) load_vector(v[k][u], src + (size_t)p[k] * stride + c.at[u]);
#pragma unroll
        for (int k = 0; k < B; ++k)
            if (whole || a + k < b)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[u][e] += v[k][u][e];
        a += B;
    };
    while (b - a >= AT) batch(std::integral_constant<int, AT>(), true);
    while (a < b) batch(std::integral_constant<int, (AT > 1 ? AT / 2 : 1)>(), false);
}

// End of the run of `key`, which holds the last position of block c and the first of block c + 1, by a wavefront: 64 blocks are tried at a time.
__device__ __forceinline__ int run_end(const int32_t* __restrict__ keys, int n, int64_t c, int key, int lane) {
    int64_t lo = c + 1, hi = (n + TOK_BLOCK - 1) / TOK_BLOCK;      // block lo begins with the key, block hi does not
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + 63) / 64, p = lo + (lane + 1) * step;
        const int t = __popcll(__ballot(p < hi && keys[p * TOK_BLOCK] == key));
        hi = min(hi, lo + (t + 1) * step);
        lo += t * step;
    }
    const int64_t i = lo * TOK_BLOCK + lane;
    return (int)(lo * TOK_BLOCK) + __popcll(__ballot(i < n && keys[i] == key));
}

// Runs, block by block, by the wavefronts of a workgroup that has positions first .. first + count - 1.
// runs: every id's run is written there.  Without it (the gradient accumulates) heads, ends: of each block, which of its positions begin a
// run, and where the run ends that holds its last one.
__device__ __forceinline__ void mark_runs(const int32_t* __restrict__ keys, int n, int rows, int64_t first, int count, TokenRun* __restrict__ runs,
                                          uint64_t* __restrict__ heads, int32_t* __restrict__ ends) {
    const int lane = threadIdx.x & 63;
    for (int w = threadIdx.x >> 6; w < count / TOK_BLOCK; w += blockDim.x >> 6) {
        const int64_t c = first / TOK_BLOCK + w, i = c * TOK_BLOCK + lane;
        if (c * TOK_BLOCK >= n) break;
        const bool in = i < n;
        const int key = in ? keys[i] : rows;
        const bool head = in && (i == 0 || keys[i - 1] != key);           // (tokens without a row have a run, too: it ends the one before)
        const bool tail = in && (i + 1 == n || keys[i + 1] != key);
        if (runs) {
            if (head && key < rows) runs[key].begin = (int)i;
            if (tail && key < rows) runs[key].end = (int)i + 1;
        } else {
            const uint64_t mask = __ballot(head);
            const int last = __builtin_amdgcn_readlane(key, 63);
            int end = (int)min((int64_t)n, (c + 1) * TOK_BLOCK);
            if (end < n && last < rows && keys[end] == last) end = run_end(keys, n, c, last, lane);
            if (lane == 0) { heads[c] = mask; ends[c] = end; }
        }
    }
}

// Zeros, one 16-byte store to a lane: of what was tried (1, 2, 4, 8 stores of a lane to a row, contiguous or not, 1 to 8 rows, workgroups that go
// round) it fills memory fastest (1 GB: 151 us, 170 to 270 us the others).  Rows of `bytes` (contiguous ones are one row); 1 << shift lanes beside one another.
struct Zeros { char* at; int64_t stride, rows, bytes; unsigned tiles; int shift; unsigned blocks; };
__device__ __forceinline__ void zero_block(const Zeros& z, unsigned block) {
    const unsigned group = block / z.tiles, tile = block - group * z.tiles;
    const int64_t row = ((int64_t)group * blockDim.x + threadIdx.x) >> z.shift, from = (((int64_t)tile << z.shift) + (threadIdx.x & ((1 << z.shift) - 1))) * 16;
    if (row >= z.rows || from >= z.bytes) return;
    typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
    char* const p = z.at + row * z.stride + from;
    if (from + 16 <= z.bytes) { *reinterpret_cast<V*>(p) = V{0, 0, 0, 0}; return; }
    for (int64_t k = 0; k < z.bytes - from; k += 2) *reinterpret_cast<uint16_t*>(p + k) = 0;
}
__global__ __launch_bounds__(TOK_THREADS) void k_token_zero(Zeros z, unsigned first) { zero_block(z, first + blockIdx.x); }
static void fill_zeros(const Zeros& z, hipStream_t st) {         // (z for TOK_THREADS)
    constexpr unsigned MOST = (unsigned)(LAUNCH_THREADS / TOK_THREADS);
    for (unsigned at = 0; at < z.blocks; at += MOST) k_token_zero<<<std::min(MOST, z.blocks - at), TOK_THREADS, 0, st>>>(z, at);
}

// all of `count` sorted positions from i are there and have one row
__device__ __forceinline__ bool one_row(const int32_t* __restrict__ keys, int n, int rows, int64_t i, int count) {
    if (i + count > n) return false;
    const int key = keys[i];
    return key < rows && keys[i + count - 1] == key;
}

// Sums of grad_out's rows by sixteens, random 256-byte to 16-KB reads: 426 k tokens of 128 16-bit columns 26 to 28 us (109 MB, 4 TB/s), 16 k of 2048 14.
// Chunks and stretches inside one run: a row-group to a chunk, 16 neighbouring ones to a stretch, whose sum they work out together; the
// chunks of such a stretch are not asked for.  Threads: 16 row-groups, or 256.  Workgroups from `blocks` on fill the gradient with zeros meanwhile.
template <int N, class S>
__global__ __launch_bounds__(1024) void k_token_chunks(Tiles q, const S* __restrict__ grad_out, int64_t stride, const int32_t* __restrict__ keys,
                                                       const int32_t* __restrict__ vals, int n, int rows, float* __restrict__ part, float* __restrict__ far,
                                                       TokenRun* __restrict__ runs, uint64_t* __restrict__ heads, int32_t* __restrict__ ends,
                                                       unsigned blocks, Zeros z) {
    extern __shared__ float chunk_lds[];
    if (blockIdx.x >= blocks) { zero_block(z, blockIdx.x - blocks); return; }
    const int groups = blockDim.x >> q.lpr_shift, lpr = 1 << q.lpr_shift;
    const Tile t = my_tile(q);
    const int64_t c = (int64_t)t.block * groups + (threadIdx.x >> q.lpr_shift);
    if (t.tile == 0) mark_runs(keys, n, rows, (int64_t)t.block * groups * TOK_CHUNK, groups * TOK_CHUNK, runs, heads, ends);
    const bool chunk = one_row(keys, n, rows, c * TOK_CHUNK, TOK_CHUNK);
    const bool stretch = chunk && one_row(keys, n, rows, c / TOK_CHUNK * TOK_STRETCH, TOK_STRETCH);
    const bool any = __syncthreads_or(stretch);
    const Cols<1> cols = my_cols<1, N>(q, t.tile);
    const int row0 = (int)c * TOK_CHUNK;
    float acc[1][N] = {};
    if (chunk && cols.at[0] >= 0) {
        add_rows<8>(acc, grad_out, stride, [=](int i) { return vals[i]; }, row0, row0 + TOK_CHUNK, cols);
        if (!stretch) store_vector(part + c * q.dim + cols.at[0], acc[0]);
    }
    if (!any) return;
    const int nt = blockDim.x;
#pragma unroll
    for (int e = 0; e < N; ++e) chunk_lds[e * nt + threadIdx.x] = acc[0][e];
    __syncthreads();
    if (!stretch) return;
    // element j of the stretch's lpr * N columns: the e-th, e = j / lpr, of lane j % lpr
    const int base = threadIdx.x & ~((TOK_CHUNK << q.lpr_shift) - 1), end = min((q.dim + N - 1) / N, (t.tile + 1) * q.per_tile);
    for (int j = threadIdx.x - base; j < lpr * N; j += TOK_CHUNK << q.lpr_shift) {
        const int e = j >> q.lpr_shift, l = j & (lpr - 1), v = t.tile * q.per_tile + l;
        if (v >= end) continue;
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < TOK_CHUNK; ++k) s += chunk_lds[e * nt + base + (k << q.lpr_shift) + l];
        far[c / TOK_CHUNK * q.dim + min(v * N, q.dim - N) + e] = s;
    }
}

// Miles inside one run, out of the stretches' sums: a row-group each.
template <int N>
__global__ __launch_bounds__(TOK_THREADS) void k_token_miles(Tiles q, const int32_t* __restrict__ keys, int n, int rows, const float* __restrict__ far,
                                                             float* __restrict__ miles) {
    const Tile t = my_tile(q);
    const int64_t m = ((int64_t)t.block * TOK_THREADS + threadIdx.x) >> q.lpr_shift;
    if (!one_row(keys, n, rows, m * TOK_MILE, TOK_MILE)) return;
    const Cols<1> cols = my_cols<1, N>(q, t.tile);
    if (cols.at[0] < 0) return;
    float acc[1][N] = {};
    add_rows<TOK_CHUNK>(acc, far, q.dim, [](int i) { return i; }, (int)m * TOK_CHUNK, ((int)m + 1) * TOK_CHUNK, cols);
    store_vector(miles + m * q.dim + cols.at[0], acc[0]);
}

struct TokenRows {
    Tiles t;
    const int32_t* vals;
    const float *part, *far, *miles;              // sums of chunks, stretches, miles (null: none are there)
    float scale;
};

// U vectors of a lane in one row of the gradient: the sum of rows, scaled, stored or added.
template <bool ADD, int U, int N, class G, class F>
__device__ __forceinline__ void token_row(float scale, G* __restrict__ out, const Cols<U>& c, F sum) {
    float acc[U][N] = {}, old[U][N];
    if (ADD) {
#pragma unroll
        for (int u = 0; u < U; ++u) if (c.at[u] >= 0) load_vector(old[u], out + c.at[u]);
        read_before_stores();
    }
    sum(acc);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (c.at[u] < 0) break;
#pragma unroll
        for (int e = 0; e < N; ++e) acc[u][e] = ADD ? fmaf(acc[u][e], scale, old[u][e]) : acc[u][e] * scale;
        store_vector(out + c.at[u], acc[u]);
    }
}

// Sorted tokens a .. b - 1, with the chunks, stretches and miles among them already summed.  token(i): the i-th sorted token.
// What lies before the first chunk and after the last is one list (two of up to 15 take a round of loads or two more), and so on upwards.
template <int U, int N, class S, class F>
__device__ __forceinline__ void add_run(float (&acc)[U][N], const TokenRows& q, const S* __restrict__ grad_out, int64_t stride, F token, int a, int b, const Cols<U>& c) {
    constexpr int AT = token_loads<U, N>;
    int c0 = (a + TOK_CHUNK - 1) / TOK_CHUNK, c1 = b / TOK_CHUNK;
    const bool parts = c0 < c1;
    {
        const int before = parts ? c0 * TOK_CHUNK - a : b - a, skip = parts ? (c1 - c0) * TOK_CHUNK : 0;
        add_rows<AT>(acc, grad_out, stride, [=](int i) { return token(a + i + (i < before ? 0 : skip)); }, 0, b - a - skip, c);
    }
    if (!parts) return;
    const float* src = q.part;
    for (int level = 0; level < 3; ++level) {
        const float* const next = level == 0 ? q.far : level == 1 ? q.miles : nullptr;
        const int s0 = (c0 + TOK_CHUNK - 1) / TOK_CHUNK, s1 = c1 / TOK_CHUNK;
        const bool more = next && s0 < s1;
        const int from = c0, before = more ? s0 * TOK_CHUNK - c0 : c1 - c0, skip = more ? (s1 - s0) * TOK_CHUNK : 0;
        add_rows<AT>(acc, src, q.t.dim, [=](int i) { return from + i + (i < before ? 0 : skip); }, 0, c1 - c0 - skip, c);
        if (!more) return;
        src = next; c0 = s0; c1 = s1;
    }
}

// Every row of the gradient, a row-group each.  (Four rows to a group, their runs read together: 595 rows of 1024 columns, 137 k tokens 106 -> 139 us, 100 k
// of 16, 65 k tokens 41 -> 47, 32,768 of 4096, 65 k tokens 343 -> 340.)
template <int U, int N, class S, class G>
__global__ __launch_bounds__(TOK_THREADS) void k_token_rows(TokenRows q, const S* __restrict__ grad_out, int64_t stride, const TokenRun* __restrict__ runs,
                                                            int rows, G* __restrict__ grad, int64_t grad_stride) {
    const Tile tile = my_tile(q.t);
    const Cols<U> cols = my_cols<U, N>(q.t, tile.tile);
    const int64_t row = ((int64_t)tile.block * TOK_THREADS + threadIdx.x) >> q.t.lpr_shift;
    if (row >= rows) return;
    const TokenRun r = runs[row];
    G* const out = grad + row * grad_stride;
    if (r.begin < 0) {
        const float none[N] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) if (cols.at[u] >= 0) store_vector(out + cols.at[u], none);
        return;
    }
    token_row<false, U, N>(q.scale, out, cols, [&](float (&acc)[U][N]) {
        add_run(acc, q, grad_out, stride, [&](int i) { return q.vals[i]; }, r.begin, r.end, cols);
    });
}

// 47 k rows of 128 columns added to, 426 k tokens 31 to 33 us; 4.7 k rows of 2048 stored, 16 k tokens 34 to 36: bound by the longest chains of loads (token, row, then up to
// 30 of each level below the last), which is why levels are sixteen apart and a group's tokens are in its lanes before it needs them.
// Rows with tokens, stored or (ADD) added to what the gradient holds: a row-group takes the runs that begin at its PER positions.
template <bool ADD, int PER, int U, int N, class S, class G>
__global__ __launch_bounds__(TOK_THREADS) void k_token_runs(TokenRows q, const S* __restrict__ grad_out, int64_t stride, const int32_t* __restrict__ keys, int n,
                                                            int rows, const uint64_t* __restrict__ heads, const int32_t* __restrict__ ends,
                                                            G* __restrict__ grad, int64_t grad_stride) {
    static_assert(TOK_BLOCK % PER == 0 && PER < 64, "positions of one block");
    const Tile tile = my_tile(q.t);
    const Cols<U> cols = my_cols<U, N>(q.t, tile.tile);
    const int64_t at = (((int64_t)tile.block * TOK_THREADS + threadIdx.x) >> q.t.lpr_shift) * PER;
    if (at >= n) return;
    const int64_t c = at / TOK_BLOCK;
    const int bit = (int)(at % TOK_BLOCK);
    const uint64_t all = heads[c];
    const int last = ends[c];
    // the positions' keys and tokens, one to a lane: read for each run as it comes up, they cost it two loads one after the other
    const int lpr = 1 << q.t.lpr_shift, lane = threadIdx.x & (lpr - 1);
    const bool held = lpr >= PER;
    const int64_t i = min(at + min(lane, PER - 1), (int64_t)n - 1);
    const int my_key = held ? keys[i] : 0, my_token = held ? q.vals[i] : 0;
    uint64_t mine = all >> bit & (((uint64_t)1 << PER) - 1);
    // Rows with one token: up to four at a time.  us a call, one by one / so: 426 k tokens of 128 added to 1 M rows 104 / 98 (popularity 1.2), 120 / 111 (1.05),
    // of 16 77 / 73, 37 k of 2048 118 / 114, 65 k of 64 59 / 55.  (Up to eight at a time: 103, 120, 72.5, 117, 55.)
    if (mine) {
        constexpr int SB = 16 / (U * N) < 2 ? 2 : 16 / (U * N) > 4 ? 4 : 16 / (U * N);
        const int head = 63 - __builtin_clzll(all);
        const uint64_t ones = (all & all >> 1) | (uint64_t)(last == (int)(c * TOK_BLOCK) + head + 1) << head;
        uint64_t left = ones >> bit & mine;
        mine &= ~left;
        while (left) {
            int key[SB], token[SB];
#pragma unroll
            for (int k = 0; k < SB; ++k) {
                const int j = left ? __builtin_ctzll(left) : 0;
                token[k] = held ? __shfl(my_token, j, lpr) : q.vals[min(at + j, (int64_t)n - 1)];
                key[k] = held ? __shfl(my_key, j, lpr) : keys[min(at + j, (int64_t)n - 1)];
                if (!left) key[k] = rows;
                left &= left - 1;
            }
            float v[SB][U][N], old[SB][U][N];
#pragma unroll
            for (int k = 0; k < SB; ++k)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (key[k] < rows && cols.at[u] >= 0) {
                        load_vector(v[k][u], grad_out + (size_t)token[k] * stride + cols.at[u]);
                        if (ADD) load_vector(old[k][u], grad + (size_t)key[k] * grad_stride + cols.at[u]);
                    }
            if (ADD) read_before_stores();
#pragma unroll
            for (int k = 0; k < SB; ++k)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (key[k] < rows && cols.at[u] >= 0) {
#pragma unroll
                        for (int e = 0; e < N; ++e) v[k][u][e] = ADD ? fmaf(v[k][u][e], q.scale, old[k][u][e]) : v[k][u][e] * q.scale;
                        store_vector(grad + (size_t)key[k] * grad_stride + cols.at[u], v[k][u]);
                    }
        }
    }
    for (; mine; mine &= mine - 1) {
        const int j = bit + __builtin_ctzll(mine);
        const uint64_t later = j < 63 ? all >> (j + 1) : 0;
        const int a = (int)(c * TOK_BLOCK) + j, b = later ? a + 1 + __builtin_ctzll(later) : last;
        const int key = held ? __shfl(my_key, a - (int)at, lpr) : keys[a];
        if (key >= rows) break;
        token_row<ADD, U, N>(q.scale, grad + (size_t)key * grad_stride, cols, [&](float (&acc)[U][N]) {
            add_run(acc, q, grad_out, stride, [&](int i) {
                const int k = i - (int)at;
                const int t = __shfl(my_token, k & (PER - 1), lpr);
                return held && k < PER ? t : q.vals[i];
            }, a, b, cols);
        });
    }
}

// Few tokens: no sort.  Every workgroup reads all ids and lists, in order, the tokens whose rows are its own: with `per_block` neighbouring rows
// to a workgroup, which also writes the zeros among them, or without (0: the gradient accumulates, or holds zeros already) as a hash of the id says.
// A row-group then goes through the list's tokens that are the first of their row, puts the row's tokens together in LDS and adds them up; the rows
// of TOK_HEAVY tokens or more are left to all row-groups together.  One launch, bound by the chain id - list - row: 1024 tokens of 100 k rows of 16 f32 columns
// with their zeros 9 to 11 us, where sort, chunks and rows take 23.
constexpr int TOK_FEW = 1024, TOK_FEW_ROWS = 1024, TOK_HEAVY = 32;
template <bool ADD, int U, int N, class S, class G, class I>
__global__ __launch_bounds__(TOK_THREADS) void k_token_few(TokenRows q, const S* __restrict__ grad_out, int64_t stride, const I* __restrict__ ids, int n, int rows,
                                                           int64_t padding_id, int per_block, unsigned blocks, G* __restrict__ grad, int64_t grad_stride,
                                                           uint32_t* flags) {
    constexpr int PER = TOK_FEW / TOK_THREADS, WAVES = TOK_THREADS / 64;
    __shared__ int list_key[TOK_FEW], list_pos[TOK_FEW], order[TOK_FEW], counts[PER * WAVES];
    __shared__ uint32_t used[TOK_FEW_ROWS / 32];
    __shared__ int heavy_row[TOK_FEW / TOK_HEAVY], heavy_from[TOK_FEW / TOK_HEAVY], heavy_count[TOK_FEW / TOK_HEAVY], heavies;
    __shared__ float sums[U * N][TOK_THREADS];
    const int lpr = 1 << q.t.lpr_shift, lane = threadIdx.x & (lpr - 1), groups = TOK_THREADS >> q.t.lpr_shift, g = threadIdx.x >> q.t.lpr_shift;
    const int w = threadIdx.x >> 6, wl = threadIdx.x & 63;
    const Tile tile = my_tile(q.t);
    const Cols<U> cols = my_cols<U, N>(q.t, tile.tile);
    const int64_t row0 = (int64_t)tile.block * per_block;
    bool bad = false;
    I id[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) id[k] = ids[min(k * TOK_THREADS + (int)threadIdx.x, n - 1)];
    if (threadIdx.x < TOK_FEW_ROWS / 32) used[threadIdx.x] = 0;
    if (threadIdx.x == 0) heavies = 0;
    int key[PER];
    uint64_t mask[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        key[k] = token_key(id[k], rows, padding_id, bad);
        const bool mine = per_block ? key[k] >= row0 && key[k] < row0 + per_block : ((unsigned)key[k] * 2654435761u >> 16) % blocks == tile.block;
        mask[k] = __ballot(mine && key[k] < rows && k * TOK_THREADS + (int)threadIdx.x < n);
        if (wl == 0) counts[k * WAVES + w] = __popcll(mask[k]);
    }
    if (bad && blockIdx.x == 0) atomicOr(flags, EF_ID_RANGE);
    __syncthreads();
    int m = 0;
    {
        int at[PER];
#pragma unroll
        for (int j = 0; j < PER * WAVES; ++j) {
            if (j % WAVES == w) at[j / WAVES] = m;
            m += counts[j];
        }
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (mask[k] >> wl & 1) {
                const int e = at[k] + __popcll(mask[k] & ((1ull << wl) - 1));
                list_key[e] = key[k];
                list_pos[e] = k * TOK_THREADS + (int)threadIdx.x;
                if (per_block) { const int r = (int)(key[k] - row0); atomicOr(&used[r / 32], 1u << r % 32); }
            }
    }
    __syncthreads();
    if (per_block) {
        const int here = (int)min((int64_t)per_block, rows - row0);
        const float none[N] = {};
        for (int r = g; r < here; r += groups) {
            if (used[r / 32] >> r % 32 & 1) continue;
#pragma unroll
            for (int u = 0; u < U; ++u) if (cols.at[u] >= 0) store_vector(grad + (row0 + r) * grad_stride + cols.at[u], none);
        }
    }
    // a lane looks at `per` neighbouring tokens of the list (an odd number, so that lanes are in different banks)
    const int per = ((m + lpr - 1) >> q.t.lpr_shift) | 1, e0 = min(m, lane * per), e1 = min(m, e0 + per);
    for (int j0 = 0; j0 < m; j0 += groups) {
        const int j = min(j0 + g, m - 1), mine = list_key[j];
        int less = 0, equal = 0, earlier = 0;
#pragma unroll 8
        for (int e = e0; e < e1; ++e) {
            const int k = list_key[e];
            less += k < mine;
            equal += k == mine;
            earlier += k == mine && e < j;
        }
        const int own = equal;
        int rank = equal;                                  // -> those of this lane and the lanes before it
        for (int o = 1; o < lpr; o <<= 1) {
            less += __shfl_xor(less, o);
            equal += __shfl_xor(equal, o);
            earlier += __shfl_xor(earlier, o);
            const int x = __shfl_up(rank, o, lpr);
            if (lane >= o) rank += x;
        }
        // (tokens of lower rows come first in `order`, so that the rows' parts of it are apart)
        const bool owner = j0 + g < m && earlier == 0;
        if (owner && own) {
            rank += less - own;
            if (equal == 1) order[rank] = list_pos[j];
            else
#pragma unroll 8
                for (int e = e0; e < e1; ++e)
                    if (list_key[e] == mine) order[rank++] = list_pos[e];
        }
        __syncthreads();
        if (!owner) continue;
        if (equal >= TOK_HEAVY && groups > 1) {
            if (lane == 0) {
                const int k = atomicAdd(&heavies, 1);
                heavy_row[k] = mine; heavy_from[k] = less; heavy_count[k] = equal;
            }
            continue;
        }
        token_row<ADD, U, N>(q.scale, grad + (size_t)mine * grad_stride, cols, [&](float (&acc)[U][N]) {
            add_rows<token_loads<U, N>>(acc, grad_out, stride, [&](int i) { return order[i]; }, less, less + equal, cols);
        });
    }
    __syncthreads();
    for (int k = 0; k < heavies; ++k) {
        const int from = heavy_from[k], end = from + heavy_count[k], share = (heavy_count[k] + groups - 1) >> (8 - q.t.lpr_shift);
        static_assert(TOK_THREADS == 256, "groups = 256 / lanes of a row");
        float acc[U][N] = {};
        add_rows<token_loads<U, N>>(acc, grad_out, stride, [&](int i) { return order[i]; }, min(end, from + g * share), min(end, from + (g + 1) * share), cols);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) sums[u * N + e][threadIdx.x] = acc[u][e];
        __syncthreads();
        if (g == 0)
            token_row<ADD, U, N>(q.scale, grad + (size_t)heavy_row[k] * grad_stride, cols, [&](float (&total)[U][N]) {
                for (int j = 0; j < groups; ++j)
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < N; ++e) total[u][e] += sums[u * N + e][(j << q.t.lpr_shift) + lane];
            });
        __syncthreads();
    }
}

// A gradient is written row by row, each once, where most rows may be in use or where it fits the memory-side cache (256 MB, with what is read);
// else zeros go everywhere first, at the rate at which memory can be filled, and the rows in use are written again.
// us a call, row by row / zeros first (16-bit rows in, f32 out; rows, columns, tokens): 131,072 x 64, 16 k 37 / 43; x 256 48 / 50; x 384 (201 MB) 60 / 65;
// x 512 (268 MB) 100 / 85; x 2048 295 / 234; 1 M x 64, 65 k 106 / 84; 1 M x 64, 1.7 M 255 / 248; 131,072 x 1024, 100 k 247 / 219; 131 k 263 / 241;
// 32,768 x 4096, 65 k 301 / 330; 16,384 x 4096, 65 k 225 / 272.  (Elements: the rows' lanes, at most two an element, fit a launch.)
static bool writes_every_row(int64_t n, int64_t rows, int64_t dim, int64_t bytes) {
    return (n >= 2 * rows && rows * dim < LAUNCH_THREADS) || bytes < (int64_t)224 << 20;
}
// Few tokens go without the sort: every row-group works out its part of the list by itself, which costs the more the wider a row is (lanes to a row-group).
// us a call, sorted / not, ids of popularity 1.05, 1.2 (16-bit rows in, f32 out): gradient of 100 k x 16, 1000 tokens 23 / 10, 22 / 13, 2000 26 / 17, 26 / 28;
// x 128, 1000 28 / 19, 28 / 28; 50 k x 512, 200 29 / 20, 31 / 22, 600 33 / 25, 34 / 35, 1000 34 / 31, 36 / 50; 8192 x 2048, 300 27 / 20, 28 / 24, 1000 30 / 35, 32 / 53;
// added to 50 k x 512, 200 22 / 19, 23 / 19, 400 24 / 20, 23 / 30.
static bool goes_unsorted(int64_t n, int dim) { return n <= TOK_FEW && n * std::min(dim, 512) <= TOK_FEW * 128; }

struct TokenWork { size_t keys, runs, heads, ends, part, far, miles, bytes; };
static TokenWork token_work(int64_t n, int64_t rows, int64_t dim) {
    TokenWork w;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t p = at; at += (bytes + 255) & ~(size_t)255; return p; };
    w.keys = take((size_t)n * 4);
    w.runs = take((size_t)rows * sizeof(TokenRun));
    w.heads = take((size_t)cdiv(n, TOK_BLOCK) * 8);
    w.ends = take((size_t)cdiv(n, TOK_BLOCK) * 4);
    w.part = take((size_t)(n / TOK_CHUNK) * dim * 4);
    w.far = take((size_t)(n / TOK_STRETCH) * dim * 4);
    w.miles = take((size_t)(n / TOK_MILE) * dim * 4);
    w.bytes = at;
    return w;
}
size_t token_work_bytes(int64_t n, int64_t rows, int64_t dim) { return token_work(n, rows, dim).bytes; }

constexpr int64_t ZEROS_BESIDE = (int64_t)512 << 20;           // bytes
static Zeros zeros_of(void* at, int64_t stride, int64_t rows, int64_t dim, int element, int threads) {
    Zeros z{(char*)at, stride * element, rows, dim * element, 1, 0, 0};
    if (stride == dim) { z.bytes *= rows; z.rows = 1; }
    z.shift = __builtin_ctz(pow2_from(cdiv(z.bytes, 16), threads));
    z.tiles = (unsigned)cdiv(z.bytes, (int64_t)16 << z.shift);
    z.blocks = (unsigned)cdiv(z.rows << z.shift, threads) * z.tiles;
    return z;
}

// f(vectors that a lane takes of a row, columns of a vector) as integral constants; wider rows go to several workgroups
template <int N, class F>
static void by_width(int dim, F f) {
    using One = std::integral_constant<int, 1>;
    if (dim < N) f(One(), One());
    else if (dim <= 64 * N || N > 4) f(One(), std::integral_constant<int, N>());
    else f(std::integral_constant<int, 2>(), std::integral_constant<int, N>());
}
// the same for kernels whose lanes take one vector
template <int N, class F>
static void by_vector(int dim, F f) {
    if (dim < N) f(std::integral_constant<int, 1>());
    else f(std::integral_constant<int, N>());
}

template <class S, class G>
static int token_bwd(fc_dense* d, const S* grad_out, int64_t stride, const int32_t* keys, int64_t n, int64_t rows, int dim, float scale, const TokenWork& w,
                     TokenRun* runs, G* grad, int64_t grad_stride, bool add) {
    const hipStream_t st = d->stream;
    int bits = 1;
    while (((int64_t)1 << bits) <= rows) ++bits;                 // keys lie in [0, rows]
    SortJob j;
    j.src = SORT_SRC_SLOTS; j.keys_in = keys; j.n = (int)n; j.num_bags = (int)n; j.one_per_bag = true; j.limit = (int)rows; j.bits = bits;
    const int32_t *ks, *vs;
    bool captured;
    FC_TRY(dense_capturing(d, &captured));
    if (captured) {
        // which of the sort's two tables is clean is known for work in order, not for a graph that is replayed: one without tables
        SortBufs& b = d->sort;
        j.keysA = b.keysA; j.valsA = b.valsA; j.keysB = b.keysB; j.valsB = b.valsB; j.ghist = b.ghist; j.dtot = b.dtot;
        FC_TRY(sort_small_fits(j) ? sort_small(j, st, &ks, &vs) : radix_sort(j, st, &ks, &vs));
    } else FC_TRY(sort_in(j, d->sort, st, &ks, &vs));
    float* part = reinterpret_cast<float*>(d->work + w.part);
    float* far = reinterpret_cast<float*>(d->work + w.far);
    float* miles = n >= TOK_MILES_FROM ? reinterpret_cast<float*>(d->work + w.miles) : nullptr;
    uint64_t* heads = reinterpret_cast<uint64_t*>(d->work + w.heads);
    int32_t* ends = reinterpret_cast<int32_t*>(d->work + w.ends);
    by_vector<VECTOR<S>>(dim, [&](auto v) {
        constexpr int N = decltype(v)::value;
        const Tiles t = tiles_of(dim, N, 1);
        const int threads = std::max(256, TOK_CHUNK << t.lpr_shift);
        const unsigned blocks = (unsigned)(cdiv(cdiv(n, TOK_CHUNK), threads >> t.lpr_shift) * t.tiles);
        // Zeros are filled in beside the chunks' sums, or, with workgroups of 1024 threads, which fill memory more slowly, by a launch of their own
        // where they take long.  us a call, own launch / beside: 131,072 x 512 (f32), 16 k tokens 92 / 85, 1 M x 64, 65 k 91 / 84, 131,072 x 2048, 16 k 227 / 234.
        Zeros z{.tiles = 1};
        if (!add && !runs) {
            z = zeros_of(grad, grad_stride, rows, dim, sizeof(G), threads);
            if ((threads > 256 && rows * dim * (int64_t)sizeof(G) > ZEROS_BESIDE) || ((int64_t)blocks + z.blocks) * threads > LAUNCH_THREADS) {
                fill_zeros(zeros_of(grad, grad_stride, rows, dim, sizeof(G), TOK_THREADS), st);
                z = Zeros{.tiles = 1};
            }
        }
        k_token_chunks<N><<<blocks + z.blocks, threads, (size_t)threads * N * 4, st>>>(t, grad_out, stride, ks, vs, (int)n, (int)rows, part, far, runs, heads, ends, blocks, z);
    });
    if (miles) by_vector<4>(dim, [&](auto v) {
        constexpr int N = decltype(v)::value;
        const Tiles t = tiles_of(dim, N, 1);
        k_token_miles<N><<<(unsigned)(cdiv((n / TOK_MILE) << t.lpr_shift, TOK_THREADS) * t.tiles), TOK_THREADS, 0, st>>>(t, ks, (int)n, (int)rows, far, miles);
    });
    by_width<VECTOR<G>>(dim, [&](auto u, auto v) {
        constexpr int U = decltype(u)::value, N = decltype(v)::value;
        const TokenRows q{tiles_of(dim, N, U), vs, part, far, miles, scale};
        auto by_runs = [&](auto a) {
            constexpr bool ADD = decltype(a)::value;
            constexpr int PER = 8;                        // us a call, 2 / 4 / 8: 426 k tokens of 128 columns added to 1 M rows 113 / 107 / 105
            k_token_runs<ADD, PER, U, N><<<(unsigned)(cdiv(cdiv(n, PER) << q.t.lpr_shift, TOK_THREADS) * q.t.tiles), TOK_THREADS, 0, st>>>(
                q, grad_out, stride, ks, (int)n, (int)rows, heads, ends, grad, grad_stride);
        };
        if (add) by_runs(std::true_type());
        else if (!runs) by_runs(std::false_type());
        else k_token_rows<U, N><<<(unsigned)(cdiv(rows << q.t.lpr_shift, TOK_THREADS) * q.t.tiles), TOK_THREADS, 0, st>>>(q, grad_out, stride, runs, (int)rows, grad, grad_stride);
    });
    FC_HIP(hipGetLastError());
    return FC_OK;
}

template <class S, class G, class I>
static int token_bwd_few(fc_dense* d, const S* grad_out, int64_t stride, const I* ids, int64_t n, int64_t rows, int dim, float scale, int64_t padding_id,
                         G* grad, int64_t grad_stride, bool add, bool zeros) {
    by_width<VECTOR<G>>(dim, [&](auto u, auto v) {
        constexpr int U = decltype(u)::value, N = decltype(v)::value;
        const TokenRows q{tiles_of(dim, N, U), nullptr, nullptr, nullptr, nullptr, scale};
        const int groups = TOK_THREADS >> q.t.lpr_shift;
        int per_block = 0;
        int64_t blocks = cdiv(n, 16);                 // lists of some 16 tokens
        if (zeros) {
            per_block = groups * (int)std::max<int64_t>(1, std::min<int64_t>(TOK_FEW_ROWS / groups, rows * q.t.tiles / (groups * 4096)));
            blocks = cdiv(rows, per_block);
        }
        const unsigned grid = (unsigned)(blocks * q.t.tiles);
        if (add) k_token_few<true, U, N><<<grid, TOK_THREADS, 0, d->stream>>>(q, grad_out, stride, ids, (int)n, (int)rows, padding_id, 0, (unsigned)blocks, grad, grad_stride, d->flags);
        else k_token_few<false, U, N><<<grid, TOK_THREADS, 0, d->stream>>>(q, grad_out, stride, ids, (int)n, (int)rows, padding_id, per_block, (unsigned)blocks, grad, grad_stride, d->flags);
    });
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
            auto run = [&](auto id) {
                using I = decltype(id);
                // Vectors of 16 bytes stored.  us a call, 16 bytes loaded / stored: f32 to bf16, 426 k rows of 128 48.4 / 39.1, 1 M of 64 58 / 46, 8192 of 4096
                // 26.2 / 23.9; f16 to f32, 24,871 of 5632 157 / 149; bf16 to f32, 100 k of 512 54.0 / 51.6, 1 M of 64 71.5 / 76.3.
                by_vector<VECTOR<D>>(dim, [&](auto v) {
                    constexpr int N = decltype(v)::value;
                    // Lanes of a row: a wavefront, or a workgroup where rows are that wide, or few.  us a call, 256 lanes / 64: 85 k rows of 206 vectors
                    // 113 / 95, 8 k of 512 18.1 / 20.7, 16 k of 1024 171 / 180.
                    // Two narrow rows to a group where there are many: one / two, 426 k of 16 vectors 21.0 / 19.5, 1 M of 16 94 / 88, 65 k of 64 16.2 / 17.1.
                    const int64_t nv = cdiv(dim, N);
                    const int sh = __builtin_ctz(pow2_from(nv, nv >= 512 || n < 2048 ? TOK_THREADS : 64));
                    auto go = [&](auto r) {
                        constexpr int ROWS = decltype(r)::value;
                        for (int64_t at = 0, most = (LAUNCH_THREADS >> sh) * ROWS; at < n; at += most) {
                            const int64_t part = std::min(most, n - at);
                            k_token_fwd<ROWS, N><<<(unsigned)cdiv(cdiv(part, ROWS) << sh, TOK_THREADS), TOK_THREADS, 0, d->stream>>>(
                                (const S*)table_dev, table_stride, (int)num_rows, dim, sh, (const I*)ids_dev + at, part, scale, (D*)out_dev + at * out_stride,
                                out_stride, d->flags);
                        }
                    };
                    if (nv <= 32 && n >= 1 << 17) go(std::integral_constant<int, 2>()); else go(std::integral_constant<int, 1>());
                });
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
        n * dim >= TOK_MOST || (id_type != FC_TYPE_I32 && id_type != FC_TYPE_I64) || !grad_table_dev || (n > 0 && (!grad_out_dev || !ids_dev)))
        return FC_ERR_INVALID_ARG;
    if (n == 0 && accumulate) return FC_OK;
    FC_HIP(hipSetDevice(d->device));
    const hipStream_t st = d->stream;
    const bool add = accumulate != 0, every_row = !add && writes_every_row(n, num_rows, dim, num_rows * dim * type_bytes(grad_table_type)), few = goes_unsorted(n, dim);
    const TokenWork w = token_work(n, every_row ? num_rows : 0, dim);
    int32_t* keys = nullptr;
    TokenRun* runs = nullptr;
    if (!few) {
        FC_TRY(dense_sort(d, n));
        FC_TRY(dense_work(d, w.bytes));
        keys = reinterpret_cast<int32_t*>(d->work + w.keys);
        if (every_row) runs = reinterpret_cast<TokenRun*>(d->work + w.runs);
        const unsigned blocks = (unsigned)cdiv(std::max<int64_t>(n, every_row ? num_rows : 0), TOK_THREADS);
        if (id_type == FC_TYPE_I32)
            k_token_keys<<<blocks, TOK_THREADS, 0, st>>>((const int32_t*)ids_dev, n, (int)num_rows, padding_id, keys, runs, d->flags);
        else k_token_keys<<<blocks, TOK_THREADS, 0, st>>>((const int64_t*)ids_dev, n, (int)num_rows, padding_id, keys, runs, d->flags);
    }
    return with_type(grad_out_type, [&](auto s) -> int {
        using S = decltype(s);
        const S* grad_out = (const S*)grad_out_dev;
        auto go = [&](auto* grad) -> int {
            if (!add && (n == 0 || (few && !every_row))) {
                fill_zeros(zeros_of(grad, grad_table_stride, num_rows, dim, sizeof(*grad), TOK_THREADS), st);
                FC_HIP(hipGetLastError());
            }
            if (!few) return token_bwd(d, grad_out, grad_out_stride, keys, n, num_rows, dim, scale, w, runs, grad, grad_table_stride, add);
            if (n > 0 && id_type == FC_TYPE_I32)
                return token_bwd_few(d, grad_out, grad_out_stride, (const int32_t*)ids_dev, n, num_rows, dim, scale, padding_id, grad, grad_table_stride, add, every_row);
            if (n > 0) return token_bwd_few(d, grad_out, grad_out_stride, (const int64_t*)ids_dev, n, num_rows, dim, scale, padding_id, grad, grad_table_stride, add, every_row);
            return FC_OK;
        };
        return grad_table_type == FC_TYPE_F32 ? go((float*)grad_table_dev) : go((S*)grad_table_dev);
    });
}

}  // extern "C"
