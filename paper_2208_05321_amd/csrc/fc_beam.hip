// Beam search: the selection over beams and vocabulary.
//
//   candidates (w, v) of a sequence:  c = s[w] + x[w, v] - log sum_u exp(x[w, u]);  of a beam that has ended only (w, eos) with c = s[w]
//   the `keep` largest, in descending order; equal ones: lower beam, larger logit, lower id
//
// Within a beam the order is that of the logits, so a slice of a row (in registers, read once) gives its `keep` largest logits and its sum of
// exponentials, and one workgroup for a sequence puts beams and slices together.  64 sequences of 8 beams of 131,072 bf16, the 16 best: 30 us for the first step, 4.5 TB/s; it reads
// each logit once and writes 8 bytes of lists a candidate.  An exponential and a comparison of each element keep the vector units busy for 49 % of that time, by their counters; wavefronts, four a SIMD, wait
// for memory or for one another for 40 % of theirs, and 31 % for their turn: loads and arithmetic hardly overlap.  The second step takes 6 us, and one sequence of 4 beams 5.2 and 3.5: what waits for one
// another there are a few accesses.
// The candidates are put in order in 64 bits.  What they are made of holds less: exponentials, and the sum of those that a lane has, are in 32 bits, and only lanes, wavefronts and slices are
// added up in 64, so that a log-sum is off by some 1e-7 (an element's exponential is one instruction in 32 bits and a function in 64).  Candidates of one beam have it in common; those of
// different beams that are closer than that may change places.
//
// The `keep` largest of a workgroup's elements: those above a bound that is no larger than the `keep`-th largest are few, and are ranked by
// counting.  The bound comes of the lanes' largest elements, by ballots, and holds the upper 16 bits of their keys: 7 bits behind the first one.  Where it does not keep all but 1024 elements of a workgroup away its
// slices are read again for each one kept, which takes milliseconds: where fewer ids than that are not masked by a finite value, where very many logits are equal, or where f32 logits lie close together for their
// size.  us, 64 sequences of 8 beams of 131,072, 16 / 64 kept: bf16 34 / 56, with all but 8 ids at -1e9 1565 / 5900, all equal 1575 / 5900; f32 with a spread of 3, 16 kept, 51, about 100 51, about 1000
// 1370, about 30,000 1640; one sequence of 4 beams, f32, 4 kept, 12.7, about 1000 19, with all but 8 ids masked, 16 kept, 38.
#include "logits_device.h"

#include <algorithm>
#include <type_traits>

namespace fc {

constexpr int BEAM_MOST = 64;                      // beams of a sequence, and candidates kept
constexpr int BEAM_LIST = 1024;                    // elements above the bound that are ranked by counting; with more of them one is found at a time

struct BeamArgs {
    const void* x;
    int64_t stride;
    const float* scores;
    const uint8_t* finished;                       // or NULL
    int32_t beams, dim, keep, eos, slices;
};
// What a slice leaves: its largest logit `from`, and its sum of 2^(c (x - from)), c = log2(e) rounded to 32 bits; its largest logits are a list of `keep`, filled up with -infinity.  A sequence's lists lie side by side, the first entries
// of all before the second ones: what neighbouring lanes of the next step hold is of different lists, and the first of a lane's is its largest, which makes its bound a good one (the other
// way round more than BEAM_LIST candidates passed it, and 5 sequences of 32 beams of 131,072 bf16, the 32 best, took 124 us, not 35).
struct BeamSlice { double sum; float from; };
struct BeamEntry { float x; uint32_t id; };        // id: and the beam, above it
constexpr int BEAM_SHIFT = 24;
static_assert(DENSE_MAX_DIM <= 1 << BEAM_SHIFT && BEAM_MOST <= 1 << (32 - BEAM_SHIFT));

// numbers in the order of unsigned integers (no distinction between zeros)
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) { return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k); }
constexpr uint32_t LOWEST = 0x00800000u;            // the lowest finite number: -infinity is no candidate
// larger logit first, then lower id
__device__ __forceinline__ uint64_t entry_key(float x, int id) { return (uint64_t)ordered(x) << 32 | (uint32_t)~id; }

template <int CTRL, int ROWS>
__device__ __forceinline__ double add_lane(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xf, false);
    return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) {
    x = add_lane<0x111, 0xf>(x);                   // row_shr 1, 2, 4, 8
    x = add_lane<0x112, 0xf>(x);
    x = add_lane<0x114, 0xf>(x);
    x = add_lane<0x118, 0xf>(x);
    x = add_lane<0x142, 0xa>(x);                   // row_bcast 15, 31
    x = add_lane<0x143, 0xc>(x);
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, 63), hi = __builtin_amdgcn_readlane((int)(u >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// The n-th largest of the wavefront's keys, but for the 16 lower bits, which are 0.
__device__ __forceinline__ uint32_t wave_bound(uint32_t key, int n) {
    uint32_t bound = 0;
#pragma unroll
    for (int b = 31; b >= 16; --b) {
        const uint32_t t = bound | 1u << b;
        if (__popcll(__ballot(key >= t)) >= n) bound = t;
    }
    return bound;
}

template <class K>
__device__ __forceinline__ K block_max(K x, K* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { const K y = __shfl_xor(x, o); x = y > x ? y : x; }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int k = 1; k < LOGIT_THREADS / 64; ++k) x = lds[k] > x ? lds[k] : x;
    __syncthreads();
    return x;
}

// whether the beam has candidates: one whose score is -infinity, or no finite number, has none
__device__ __forceinline__ bool beam_lives(const BeamArgs& a, int64_t row) {
    const float s = a.scores[row];
    return s - s == 0.f;
}

// `run` neighbouring slices of a row, one after the other.  Of each wavefront's lanes the largest elements so far give a bound that a quarter of `keep` of them reach; the least of
// the four is reached by `keep` elements.  (The `keep`-th of one wavefront's is a bound as well, and four times as many elements are above it.)  After the first slice a
// wavefront looks at the bounds when it meets elements above its own; what the others have come to meanwhile does not matter, as bounds only rise.
template <class T, int PER>
__global__ __launch_bounds__(LOGIT_THREADS) void k_beam_slice(BeamArgs a, int64_t first, int run, BeamSlice* __restrict__ sums, BeamEntry* __restrict__ lists) {
    using Slice = RowSlice<T, LOGIT_THREADS, PER>;
    constexpr int N = Slice::N, WAVES = LOGIT_THREADS / 64;
    __shared__ uint64_t list[BEAM_LIST], few[BEAM_LIST];
    __shared__ uint64_t best[WAVES];
    __shared__ float froms[WAVES];
    __shared__ double parts[WAVES];
    __shared__ uint32_t bounds[WAVES];
    __shared__ int count, kept;
    const int lane = threadIdx.x, part = blockIdx.x % a.slices, begin = part * run * Slice::COLUMNS;
    const int64_t local = blockIdx.x / a.slices, row = first + local;
    const uint32_t all = a.beams * a.slices, seq = blockIdx.x / all, beam = (uint32_t)(local - seq * a.beams) << BEAM_SHIFT;
    BeamEntry* out = lists + (int64_t)seq * all * a.keep + (blockIdx.x - seq * all);
    const bool lives = beam_lives(a, row);
    if (!lives || (a.finished && a.finished[row])) {             // no candidate, or the end again
        for (int i = lane; i < a.keep; i += LOGIT_THREADS) out[i * all] = lives && part == 0 && i == 0 ? BeamEntry{0.f, beam | (uint32_t)a.eos} : BeamEntry{-INFINITY, 0};
        return;
    }
    const T* x = (const T*)a.x + row * a.stride;
    const int end = (int)min((int64_t)a.dim, begin + (int64_t)run * Slice::COLUMNS);
    Slice s;
    s.load(x, begin, lane, a.dim, true);
    if (lane == 0) count = kept = 0;
    auto bound = [&]() {
        uint32_t b = __hip_atomic_load(&bounds[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
#pragma unroll
        for (int k = 1; k < WAVES; ++k) b = min(b, __hip_atomic_load(&bounds[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
        return max(b, LOWEST);
    };
    float lane_top = -INFINITY, sum = 0.f, least = -INFINITY;
    for (int base = begin; base < end; base += Slice::COLUMNS) {
        const int lane = here(threadIdx.x);
        if (base > begin) s.load_long(x, base, lane, a.dim, true);
        s.cut(base, lane, a.dim);
        const float top = s.largest();
        s.forget();
        // sum of exponentials, each lane's from its own largest element so far
        const float to = fmaxf(lane_top, top);
        const Exponents f = exponents(to, LOG2E);
        sum = sum * part_of(lane_top, to, LOG2E) + s.exponentials(f.scale, f.off) * f.back;
        lane_top = to;
        if (base > begin && !__any(top >= least)) continue;
        const uint32_t mine = wave_bound(ordered(lane_top), (a.keep + WAVES - 1) / WAVES);
        if ((lane & 63) == 0) __hip_atomic_store(&bounds[lane >> 6], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        if (base == begin) __syncthreads();
        uint32_t key = bound();
        if (key == LOWEST) key = max(key, wave_bound(ordered(lane_top), a.keep));      // (a wavefront without elements: the own one's bound, if it has one)
        least = unordered(key);
        if (!(top >= least)) continue;
        s.forget();
        uint32_t at = s.vectors_from(least);
        while (at) {
            const int k = __builtin_ctz(at);
            at &= at - 1;
            const typename Slice::V v = s.pick(k);
            const int col = min(Slice::column(base, lane, k), a.dim - N);
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) hits |= (float)v[e] >= least ? 1u << e : 0;
            while (hits) {
                const int e = __builtin_ctz(hits);
                hits &= hits - 1;
                float f = (float)v[0];
#pragma unroll
                for (int j = 1; j < N; ++j) { const float y = (float)v[j]; f = j == e ? y : f; }
                const int p = atomicAdd(&count, 1);
                if (p < BEAM_LIST) list[p] = entry_key(f, col + e);
            }
        }
    }
    const float from_wave = wave_max(lane_top);
    const double sum_wave = wave_sum((double)(sum * part_of(lane_top, from_wave, LOG2E)));
    if ((lane & 63) == 0) { froms[lane >> 6] = from_wave; parts[lane >> 6] = sum_wave; }
    __syncthreads();
    auto put = [&](int at, uint64_t key) { out[at * all] = BeamEntry{unordered((uint32_t)(key >> 32)), beam | ~(uint32_t)key}; };
    const uint64_t lowest = (uint64_t)bound() << 32;
    if (count <= BEAM_LIST) {
        for (int i = lane; i < count; i += LOGIT_THREADS) {
            const uint64_t key = list[i];
            if (key >= lowest) few[atomicAdd(&kept, 1)] = key;
        }
        __syncthreads();
        const int got = kept;
        for (int i = lane >> 3; i < got; i += LOGIT_THREADS / 8) {   // eight lanes to an element
            const uint64_t key = few[i];
            int rank = 0;
            for (int j = lane & 7; j < got; j += 8) rank += few[j] > key;
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) rank += __shfl_xor(rank, o);
            if (rank < a.keep && (lane & 7) == 0) put(rank, key);
        }
        for (int i = got + lane; i < a.keep; i += LOGIT_THREADS) out[i * all] = BeamEntry{-INFINITY, 0};
    } else {                                       // (more than BEAM_LIST have the key's upper bits in common with the least of those that are kept)
        uint64_t last = ~0ull;
        for (int i = 0; i < a.keep; ++i) {
            uint64_t mine = 0;
            for (int c = begin + lane; c < end; c += LOGIT_THREADS) {
                const float v = (float)x[c];
                const uint64_t key = entry_key(v, c);
                if (v == v && key >= lowest && key < last && key > mine) mine = key;
            }
            last = block_max(mine, best);
            if (lane == 0) put(i, last);
        }
    }
    if (lane == 0) {
        float to = froms[0];
        for (int k = 1; k < WAVES; ++k) to = fmaxf(to, froms[k]);
        double total = 0.;
        for (int k = 0; k < WAVES; ++k) total += parts[k] * (double)part_of(froms[k], to, LOG2E);
        sums[blockIdx.x] = BeamSlice{total, to};
    }
}

// A candidate in the order of the search.
struct Candidate { double c; float x; int32_t beam, id; };
__device__ __forceinline__ bool before(const Candidate& p, const Candidate& q) {
    if (p.c != q.c) return p.c > q.c;
    if (p.beam != q.beam) return p.beam < q.beam;
    if (p.x != q.x) return p.x > q.x;
    return p.id < q.id;
}

constexpr int JOIN_THREADS = 512;
// Entries that a lane holds in registers; those of larger searches are read again (all of them read again: one sequence of 4 beams of 131,072 ids, alone, 30.7 us, not 28.1; 64 of 8 as fast).
constexpr int JOIN_HELD = 4;
// Candidates above the bound beyond which a higher one is looked for: to rank 1024 takes some 40 us.  us, at 256 / 512 / 1024: one sequence of 32 beams of 131,072 bf16, the 64 best
// 44.5 / 49.7 / 86.8, one of one beam of 250,000 29 / 80 / 80.
constexpr int JOIN_FEW = 256;

// One workgroup puts a sequence's beams and slices together.  Everything it needs is asked for at once; what follows are a few steps that wait for one another (one sequence of 4
// beams of 131,072 ids 13.4 us when lists were read after their lengths and the bound was found by comparing all lanes, 3.7 this way; 64 sequences of 8 beams 21.4 and 6.2).
template <bool HELD>
__global__ __launch_bounds__(JOIN_THREADS) void k_beam_join(BeamArgs a, int64_t first, const BeamSlice* __restrict__ sums, const BeamEntry* __restrict__ lists,
                                                            float* __restrict__ scores_out, int32_t* __restrict__ parents_out, void* __restrict__ tokens_out,
                                                            int32_t token_type, uint8_t* __restrict__ finished_out) {
    constexpr int WAVES = JOIN_THREADS / 64;
    __shared__ double add[BEAM_MOST];              // what a beam's logits, less its largest, lack to be candidates; not finite: there are none
    __shared__ double tops[BEAM_MOST];             // their largest (far from zero the log-sum itself would be lost in its sum with that); in 64 bits, which saves a conversion a candidate
    __shared__ uint32_t bounds[WAVES], shares[WAVES], highs[WAVES];
    __shared__ double list_c[BEAM_LIST];           // and bins
    __shared__ Candidate list[BEAM_LIST];
    __shared__ int count;
    const int lane = threadIdx.x;
    const int64_t seq = blockIdx.x, row0 = first + seq * a.beams;
    const int all = a.beams * a.slices * a.keep;                    // (below 2^22)
    const BeamEntry* entries = lists + seq * all;
    BeamEntry held[JOIN_HELD];
    if constexpr (HELD) {
#pragma unroll
        for (int j = 0; j < JOIN_HELD; ++j) held[j] = entries[min(lane + j * JOIN_THREADS, all - 1)];
    }
    for (int w = lane >> 6; w < a.beams; w += WAVES) {
        const BeamSlice* s = sums + (seq * a.beams + w) * a.slices;
        BeamSlice q = s[min(lane & 63, a.slices - 1)];              // (of a beam without candidates: whatever the workspace holds, not used)
        const float score = a.scores[row0 + w];
        const bool lives = score - score == 0.f, end = a.finished && a.finished[row0 + w];
        double v = lives ? 0. : -INFINITY;
        float top = 0.f;
        if (lives && !end) {
            if ((lane & 63) >= a.slices) q = BeamSlice{0., -INFINITY};
            for (int k = (lane & 63) + 64; k < a.slices; k += 64) {
                const BeamSlice o = s[k];
                const float to = fmaxf(q.from, o.from);
                q.sum = q.sum * (double)part_of(q.from, to, LOG2E) + o.sum * (double)part_of(o.from, to, LOG2E);
                q.from = to;
            }
            top = from_of(wave_max(q.from));
            v = -log2(wave_sum(q.sum * (double)part_of(q.from, top, LOG2E))) / (double)LOG2E;      // (the constant that the exponents were made with: what it is off by cancels)
        }
        if ((lane & 63) == 0) { add[w] = v + (double)score; tops[w] = (double)top; }
    }
    if (lane == 0) count = 0;
    __syncthreads();
    // f(candidate) for each of this lane's candidates; whether it is one to consider, or any later one of its list.  All lanes come here together.
    auto candidates = [&](auto f) {
        bool used;
        auto one = [&](const BeamEntry& e) {
            if (e.x == -INFINITY) return;
            const int w = e.id >> BEAM_SHIFT;
            const double v = add[w];
            if (v - v == 0.) used |= f(Candidate{((double)e.x - tops[w]) + v, e.x, w, (int32_t)(e.id & ((1u << BEAM_SHIFT) - 1))});
        };
        if constexpr (HELD) {
            used = false;
#pragma unroll
            for (int j = 0; j < JOIN_HELD; ++j) if (lane + j * JOIN_THREADS < all) one(held[j]);
        } else {
            int idle = 0;                          // entries one after the other that f had no use for: of every list one, if there are as many as lists, and what follows in them is lower
            for (int i = lane; i - lane < all && idle < a.beams * a.slices; i += JOIN_THREADS * JOIN_HELD) {
                BeamEntry e[JOIN_HELD];
#pragma unroll
                for (int j = 0; j < JOIN_HELD; ++j) e[j] = entries[min(i + j * JOIN_THREADS, all - 1)];
                used = false;
#pragma unroll
                for (int j = 0; j < JOIN_HELD; ++j) if (i + j * JOIN_THREADS < all) one(e[j]);
                idle = __syncthreads_or(used) ? 0 : idle + JOIN_THREADS * JOIN_HELD;
            }
        }
    };
    // Bounds are keys of candidates rounded to 32 bits, which keeps their order.  Two that `keep` candidates reach: the `keep`-th of a wavefront's lanes' largest, and the least of what
    // an eighth of `keep` of each wavefront's reach.  (Lanes without a candidate count as the lowest key.)
    auto key_of = [](double c) { return ordered((float)c); };
    double top = -INFINITY;
    candidates([&](const Candidate& q) { const bool more = q.c > top; top = fmax(top, q.c); return more; });
    const uint32_t top_key = key_of(top), mine = wave_bound(top_key, a.keep), share = wave_bound(top_key, (a.keep + WAVES - 1) / WAVES);
    const float high = wave_max((float)top);
    if ((lane & 63) == 0) { bounds[lane >> 6] = mine; shares[lane >> 6] = share; highs[lane >> 6] = ordered(high); }
    __syncthreads();
    uint32_t low = shares[0], hi = highs[0];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) { low = min(low, shares[k]); hi = max(hi, highs[k]); }
#pragma unroll
    for (int k = 0; k < WAVES; ++k) low = max(low, bounds[k]);
    auto collect = [&]() {                         // what is above the bound, and how many
        candidates([&](const Candidate& q) {
            if (key_of(q.c) < low) return false;
            const int p = atomicAdd(&count, 1);
            if (p < BEAM_LIST) { list_c[p] = q.c; list[p] = q; }
            return true;
        });
        __syncthreads();
        return count;
    };
    int got = collect();
    if (got > JOIN_FEW) {                          // a higher bound: the keys above this one are counted in 1024 bins, and the bin of the `keep`-th in as many again
        uint32_t* bins = reinterpret_cast<uint32_t*>(list_c);
        constexpr int BINS = 1024, EACH = BINS / 64;
        int shift = 1;
        while (got > JOIN_FEW && shift > 0 && hi > low) {
            shift = max(0, 22 - __builtin_clz(hi - low));
            __syncthreads();
            for (int i = lane; i < BINS; i += JOIN_THREADS) bins[i] = 0;
            __syncthreads();
            candidates([&](const Candidate& q) {
                const uint32_t k = key_of(q.c);
                if (k >= low) atomicAdd(&bins[min((k - low) >> shift, BINS - 1u)], 1u);
                return k >= low;
            });
            __syncthreads();
            if (lane < 64) {                       // each lane has EACH bins, the first lane the highest ones
                const uint32_t* own = bins + (63 - lane) * EACH;
                int sum = 0;
                for (int i = 0; i < EACH; ++i) sum += (int)own[i];
                int upto = sum;
                for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(upto, o); if (lane >= o) upto += y; }
                if (upto >= a.keep && upto - sum < a.keep) {
                    int n = upto - sum, i = EACH;
                    while (n < a.keep) n += (int)own[--i];
                    bounds[0] = low + ((uint32_t)((63 - lane) * EACH + i) << shift);
                    count = n;
                }
            }
            __syncthreads();
            low = bounds[0];
            got = count;
            hi = min(hi, low + (1u << shift) - 1);
        }
        if (got <= BEAM_LIST) {
            __syncthreads();
            if (lane == 0) count = 0;
            __syncthreads();
            got = collect();
        }
    }
    auto put = [&](int at, const Candidate& q) {
        const int64_t o = seq * a.keep + at;
        scores_out[o] = (float)q.c;
        parents_out[o] = q.beam;
        if (token_type == FC_TYPE_I64) ((int64_t*)tokens_out)[o] = q.id; else ((int32_t*)tokens_out)[o] = q.id;
        if (finished_out) finished_out[o] = q.id == a.eos;
    };
    if (got <= BEAM_LIST) {
        for (int i = lane >> 3; i < got; i += JOIN_THREADS / 8) {    // eight lanes to a candidate
            const double c = list_c[i];
            int rank = 0;
            for (int j = lane & 7; j < got; j += 8) {
                const double o = list_c[j];
                if (o > c || (o == c && j != i && before(list[j], list[i]))) ++rank;
            }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) rank += __shfl_xor(rank, o);
            if (rank < a.keep && (lane & 7) == 0) put(rank, list[i]);
        }
        got = min(got, a.keep);
    } else {                                       // (over BEAM_LIST candidates that are equal in 32 bits)
        Candidate last{INFINITY, 0.f, -1, -1};
        got = a.keep;
        for (int i = 0; i < a.keep; ++i) {
            Candidate mine{-INFINITY, 0.f, 1 << 30, 0};
            candidates([&](const Candidate& q) { if (before(last, q) && before(q, mine)) mine = q; return key_of(q.c) >= low; });
            __syncthreads();
            list[lane] = mine;
            for (int o = JOIN_THREADS / 2; o > 0; o >>= 1) {
                __syncthreads();
                if (lane < o && before(list[lane + o], list[lane])) list[lane] = list[lane + o];
            }
            __syncthreads();
            last = list[0];
            if (lane == 0) put(i, last);
        }
    }
    for (int i = got + lane; i < a.keep; i += JOIN_THREADS) put(i, Candidate{-INFINITY, 0.f, 0, max(a.eos, 0)});
}

// Workgroups of the first step, beyond which they take several slices each, up to 8: the bound is found once, and is high already for the later ones.  us, at 512 / 1024 / 2048 workgroups /
// one slice each: 64 sequences of 8 beams of 131,072 bf16 36.7 / 32.3 / 33.4 / 35.7.
constexpr int64_t BEAM_GROUPS = 1024;
constexpr size_t BEAM_WORK = (size_t)5 << 20;      // of a launch's slices (one sequence takes 4.4 MB at most); more sequences go in several
size_t beam_work_bytes() { return BEAM_WORK; }

template <class T, int PER>
void beam_run(fc_dense* d, BeamArgs a, int64_t batch, float* scores, int32_t* parents, void* tokens, int32_t token_type, uint8_t* finished) {
    const int64_t slices = cdiv(a.dim, RowSlice<T, LOGIT_THREADS, PER>::COLUMNS), run = std::clamp<int64_t>(batch * a.beams * slices / BEAM_GROUPS, 1, 8);
    a.slices = (int32_t)cdiv(slices, run);
    const size_t of_seq = (size_t)a.beams * a.slices * (sizeof(BeamSlice) + a.keep * sizeof(BeamEntry));
    const int64_t most = std::max<int64_t>(1, (int64_t)(BEAM_WORK / of_seq));
    for (int64_t at = 0; at < batch; at += most) {
        const int64_t n = std::min(most, batch - at);
        BeamSlice* sums = reinterpret_cast<BeamSlice*>(d->work);
        BeamEntry* lists = reinterpret_cast<BeamEntry*>(sums + n * a.beams * a.slices);
        k_beam_slice<T, PER><<<(unsigned)(n * a.beams * a.slices), LOGIT_THREADS, 0, d->stream>>>(a, at * a.beams, (int)run, sums, lists);
        const int64_t o = at * a.keep;
        auto join = [&](auto held) {
            k_beam_join<decltype(held)::value><<<(unsigned)n, JOIN_THREADS, 0, d->stream>>>(a, at * a.beams, sums, lists, scores + o, parents + o,
                                                                                           (char*)tokens + o * (token_type == FC_TYPE_I64 ? 8 : 4), token_type, finished ? finished + o : nullptr);
        };
        if (a.beams * a.slices * a.keep <= JOIN_THREADS * JOIN_HELD) join(std::true_type()); else join(std::false_type());
    }
}

}  // namespace fc

using namespace fc;

extern "C" {

int beam_select(fc_dense* d, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t batch, int32_t beams, int32_t dim, const float* scores_dev,
                const uint8_t* finished_dev, int32_t eos_id, int32_t keep, float* scores_out_dev, int32_t* parents_out_dev, void* tokens_out_dev, int32_t token_type,
                uint8_t* finished_out_dev) {
    if (!d || batch < 0 || batch >= DENSE_LIMIT || beams <= 0 || beams > BEAM_MOST || keep <= 0 || keep > BEAM_MOST || dim <= 0 || dim > DENSE_MAX_DIM || logits_stride < dim ||
        !is_float_type(type) || (token_type != FC_TYPE_I32 && token_type != FC_TYPE_I64) || eos_id < -1 || eos_id >= dim || (finished_dev && eos_id < 0) ||
        (finished_out_dev && eos_id < 0) || (batch > 0 && (!logits_dev || !scores_dev || !scores_out_dev || !parents_out_dev || !tokens_out_dev)))
        return FC_ERR_INVALID_ARG;
    if (batch == 0) return FC_OK;
    FC_HIP(hipSetDevice(d->device));
    FC_TRY(dense_work(d, BEAM_WORK));
    return with_type(type, [&](auto t) -> int {
        using T = decltype(t);
        const BeamArgs a{logits_dev, logits_stride, scores_dev, finished_dev, beams, dim, keep, eos_id, 1};
        const int64_t vectors = cdiv(dim, VECTOR<T>);
        // Vectors of a lane: 8, or 2 where slices of 8 are too few to keep all compute units reading.  us, 8 / 2: 64 sequences of 8 beams of 131,072 bf16 33.5 / 40.8, 33 of 5 of 50,021 f32
        // 15.4 / 17.1, but one of 4 beams of 131,072, alone, 29.4 / 28.0.  Not for long lists, as there are four times as many then: one of 32 beams, the 64 best, 36.7 / 44.5.
        if (vectors <= LOGIT_THREADS * 2 || (keep <= 16 && batch * beams * cdiv(vectors, LOGIT_THREADS * 8) < 512))
            beam_run<T, 2>(d, a, batch, scores_out_dev, parents_out_dev, tokens_out_dev, token_type, finished_out_dev);
        else beam_run<T, 8>(d, a, batch, scores_out_dev, parents_out_dev, tokens_out_dev, token_type, finished_out_dev);
        FC_HIP(hipGetLastError());
        return FC_OK;
    });
}

}  // extern "C"
