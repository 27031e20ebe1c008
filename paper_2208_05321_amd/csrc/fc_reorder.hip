// Reordering of the states of beams: row (b, j) becomes row (b, parent[b, j]), for a list of tensors, in place or into others.
//
// A copy, bound by HBM: what is read are the distinct parents of the rows that change, what is written those rows.  A thread owns 16 bytes of every beam's row of a
// sequence (8 or 4 where there are more than 16 or 32 of them) and reads all of them before it writes one, so that in place a row may be another's
// source in any pattern, without a second buffer or a wait between workgroups.  Rows that stay are not touched.  16 sequences of 8 beams, 24 tensors of 512 KB a row in
// place (2.3 GB that must move): 435 us, 5.4 TB/s.
#include "dense_device.h"

#include <algorithm>
#include <type_traits>

namespace fc {

constexpr int STATE_THREADS = 256;
constexpr int STATE_MOST_BEAMS = 64;
constexpr int STATE_GROUP = 44;                    // tensors that one launch's arguments can describe
// Vectors of 16 bytes of a row that a workgroup moves, for every beam.  us, 64 / 128 / 256 / 512 / 1024: 16 sequences of 8 beams, 24 tensors of 512 KB a row in place 458 / 433 / 440 / 449 / 457, one
// sequence of 4 beams (17 tensors of 30 KB; host) 20.4 each.
constexpr int STATE_TILE = 256;
struct StateRows {
    const char* src;
    char* dst;
    int64_t src_row, dst_row, src_piece, dst_piece, begin;      // begin: its first workgroup
    uint32_t piece, vectors;                       // bytes of a piece; vectors of a row (pieces * those of a piece)
    uint32_t per, tiles;                           // vectors of a piece, workgroups of a sequence
};
struct StateGroup { StateRows t[STATE_GROUP]; int count; };
static_assert(sizeof(StateGroup) + 64 <= 4096, "arguments of a launch");

template <int BYTES> struct Chunk { typedef uint32_t V __attribute__((ext_vector_type(BYTES / 4), aligned(1))); };
template <> struct Chunk<4> { typedef uint32_t V __attribute__((aligned(1))); };
template <> struct Chunk<2> { typedef uint16_t V __attribute__((aligned(1))); };
template <> struct Chunk<1> { typedef uint8_t V; };

struct Moves { int64_t from[STATE_MOST_BEAMS], to[STATE_MOST_BEAMS]; int count, none; };   // in bytes; none: rows that become zeros, listed from the end of `to`
__device__ __forceinline__ int64_t same(int64_t x) {          // of a number that all lanes have: in scalar registers
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// Moves [begin, begin + n) of one chunk of the rows: all rows are read before one is written, as in place a row may be another's source.
template <int BYTES, int MOST>
__device__ __forceinline__ void move_chunk(const char* src, char* dst, const Moves& m, int begin, int n, bool stream) {
    typename Chunk<BYTES>::V v[MOST];
#pragma unroll
    for (int i = 0; i < MOST; ++i)
        v[i] = *reinterpret_cast<const typename Chunk<BYTES>::V*>(src + same(m.from[begin + min(i, n - 1)]));
    using V = typename Chunk<BYTES>::V;
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < MOST; ++i)
            if (i < n) f(i, dst + same(m.to[begin + i]));
    };
    if (stream) apart<1>([&] { each([&](int i, char* o) { __builtin_nontemporal_store(v[i], reinterpret_cast<V*>(o)); }); });
    else apart<0>([&] { each([&](int i, char* o) { *reinterpret_cast<V*>(o) = v[i]; }); });
}
template <int BYTES, int MOST>
__device__ __forceinline__ void move_rows(const char* src, char* dst, const Moves& m, bool stream) {
    const int count = __builtin_amdgcn_readfirstlane(m.count);
    for (int k = 0; k < count; k += MOST) move_chunk<BYTES, MOST>(src, dst, m, k, min(MOST, count - k), stream);
    for (int i = 0; i < m.none; ++i) *reinterpret_cast<typename Chunk<BYTES>::V*>(dst + same(m.to[STATE_MOST_BEAMS - 1 - i])) = typename Chunk<BYTES>::V{};
}
template <int MOST>
__device__ __forceinline__ void move_tile(const StateRows& t, const char* src, char* dst, int tile, const Moves& m, bool stream) {
    constexpr int BYTES = MOST <= 16 ? 16 : MOST <= 32 ? 8 : 4, SPLIT = 16 / BYTES;       // 64 registers of a lane at most
    for (uint32_t i = threadIdx.x; i < STATE_TILE * SPLIT; i += STATE_THREADS) {
        const uint32_t v = (uint32_t)tile * STATE_TILE + i / SPLIT;
        if (v >= t.vectors) break;
        const uint32_t piece = t.per == t.vectors ? 0 : v / t.per;
        uint32_t at = (v - piece * t.per) * 16 + i % SPLIT * BYTES;
        const char* s = src + piece * t.src_piece;
        char* o = dst + piece * t.dst_piece;
        if (at + BYTES <= t.piece) { move_rows<BYTES, MOST>(s + at, o + at, m, stream); continue; }
        if (at >= t.piece) continue;
        const uint32_t left = t.piece - at;
        if (BYTES > 8 && left & 8) { move_rows<8, MOST>(s + at, o + at, m, stream); at += 8; }
        if (BYTES > 4 && left & 4) { move_rows<4, MOST>(s + at, o + at, m, stream); at += 4; }
        if (left & 2) { move_rows<2, MOST>(s + at, o + at, m, stream); at += 2; }
        if (left & 1) move_rows<1, MOST>(s + at, o + at, m, stream);
    }
}

// MOST: moves of a sequence that go at once: all of them where they are in place, else eight.
template <int MOST>
__global__ __launch_bounds__(STATE_THREADS) void k_beam_reorder(StateGroup g, int64_t first, bool stream, const void* __restrict__ parents, int32_t parent_type, int beams, int keep,
                                                                uint32_t* __restrict__ flags) {
    __shared__ Moves m;
    const int64_t block = first + blockIdx.x;
    int lo = 0, hi = g.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (g.t[mid].begin <= block) lo = mid; else hi = mid;
    }
    const StateRows& t = g.t[lo];
    const int64_t seq = (block - t.begin) / t.tiles;
    const int tile = (int)((block - t.begin) - seq * t.tiles);
    const bool in_place = t.src == t.dst;
    if (threadIdx.x < 64) {
        const int j = threadIdx.x;
        int64_t p = -1;
        if (j < keep) p = parent_type == FC_TYPE_I64 ? ((const int64_t*)parents)[seq * keep + j] : (int64_t)((const int32_t*)parents)[seq * keep + j];
        const bool known = p >= 0 && p < beams;
        if (j < keep && !known) atomicOr(flags, (uint32_t)EF_ID_RANGE);
        const bool moves = known && !(in_place && p == j), none = j < keep && !known && !in_place;
        const uint64_t mm = __ballot(moves), nn = __ballot(none), below = ((uint64_t)1 << j) - 1;
        if (moves) { const int k = __popcll(mm & below); m.from[k] = p * t.src_row; m.to[k] = j * t.dst_row; }
        if (none) m.to[STATE_MOST_BEAMS - 1 - __popcll(nn & below)] = j * t.dst_row;
        if (j == 0) { m.count = __popcll(mm); m.none = __popcll(nn); }
    }
    __syncthreads();
    const char* src = t.src + seq * beams * t.src_row;
    char* dst = t.dst + seq * keep * t.dst_row;
    move_tile<MOST>(t, src, dst, tile, m, stream);
}

}  // namespace fc

using namespace fc;

extern "C" {

int beam_reorder(fc_dense* d, const fc_state* states, int32_t count, int64_t batch, int32_t beams, const void* parents_dev, int32_t parent_type, int32_t keep) {
    if (!d || count < 0 || batch < 0 || batch >= DENSE_LIMIT || beams <= 0 || beams > STATE_MOST_BEAMS || keep <= 0 || keep > STATE_MOST_BEAMS ||
        (parent_type != FC_TYPE_I32 && parent_type != FC_TYPE_I64) || (count > 0 && !states) || (count > 0 && batch > 0 && !parents_dev))
        return FC_ERR_INVALID_ARG;
    for (int32_t k = 0; k < count; ++k) {
        const fc_state& s = states[k];
        if (s.piece_bytes < 0 || s.pieces < 0) return FC_ERR_INVALID_ARG;
        if (s.piece_bytes == 0 || s.pieces == 0 || batch == 0) continue;
        if (!s.src || !s.dst || s.dst == parents_dev || s.pieces >= (int64_t)1 << 31 || s.piece_bytes >= (int64_t)1 << 31 || cdiv(s.piece_bytes, 16) * s.pieces >= (int64_t)1 << 31 ||
            (s.pieces > 1 && (s.src_piece < s.piece_bytes || s.dst_piece < s.piece_bytes)) ||
            s.src_row < (s.pieces - 1) * s.src_piece + s.piece_bytes || s.dst_row < (s.pieces - 1) * s.dst_piece + s.piece_bytes ||
            (s.src == s.dst && (keep != beams || s.src_row != s.dst_row || (s.pieces > 1 && s.src_piece != s.dst_piece))))
            return FC_ERR_INVALID_ARG;
    }
    if (batch == 0) return FC_OK;
    FC_HIP(hipSetDevice(d->device));
    int64_t bytes = 0;
    bool in_place = false;
    for (int32_t k = 0; k < count; ++k) {
        bytes += states[k].piece_bytes * states[k].pieces * batch * keep;
        in_place |= states[k].src == states[k].dst;
    }
    // What the memory-side cache would not hold until it is read is stored past it.  us, stores through / past the caches, rows of 512 KB in place: 32 MB 19.5 / 19.8, 64 MB 42.8 / 36.1, 128 MB 79.6 / 76.8, 192 MB
    // 115.9 / 112.5, 512 MB 306 / 299; into others 26.3 / 26.4, 44.6 / 38.1, 83.0 / 76.9, 119.4 / 111.2, 324 / 304: below 128 MB the line goes by the next reader, who finds them there.  (Loads past the caches as
    // well, beyond 128 MB: into others 3 % more, as a row may have several takers; in place 9 % less, 440 / 401 for 1.6 GB of 24 tensors, which is not made use of.)
    const bool stream = bytes > (int64_t)128 << 20;
    StateGroup g;
    g.count = 0;
    int64_t blocks = 0;
    auto launch = [&]() {
        const int64_t most = LAUNCH_THREADS / STATE_THREADS;
        auto go = [&](auto moves) {
            for (int64_t at = 0; at < blocks; at += most)
                k_beam_reorder<decltype(moves)::value><<<(unsigned)std::min(most, blocks - at), STATE_THREADS, 0, d->stream>>>(g, at, stream, parents_dev, parent_type, beams, keep,
                                                                                                                              d->flags);
        };
        if (!in_place || keep <= 8) go(std::integral_constant<int, 8>());
        else if (keep <= 16) go(std::integral_constant<int, 16>());
        else if (keep <= 32) go(std::integral_constant<int, 32>());
        else go(std::integral_constant<int, 64>());
        g.count = 0;
        blocks = 0;
    };
    for (int32_t k = 0; k < count; ++k) {
        fc_state s = states[k];
        if (s.piece_bytes == 0 || s.pieces == 0) continue;
        if (s.pieces > 1 && s.src_piece == s.piece_bytes && s.dst_piece == s.piece_bytes && s.pieces * s.piece_bytes < (int64_t)1 << 31) {
            s.piece_bytes *= s.pieces;             // neighbours are one piece
            s.pieces = 1;
        }
        if (g.count == STATE_GROUP) launch();
        const int64_t per = cdiv(s.piece_bytes, 16), tiles = cdiv(per * s.pieces, STATE_TILE);
        g.t[g.count++] = StateRows{(const char*)s.src, (char*)s.dst, s.src_row, s.dst_row, s.src_piece, s.dst_piece, blocks, (uint32_t)s.piece_bytes,
                                   (uint32_t)(per * s.pieces), (uint32_t)per, (uint32_t)tiles};
        blocks += tiles * batch;
    }
    launch();
    FC_HIP(hipGetLastError());
    return FC_OK;
}

}  // extern "C"
