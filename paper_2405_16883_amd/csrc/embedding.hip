// Lookup of rows by token id, and the gradient of the table it reads.
//
// Lookup: out[t, :] = scale E[ids[t], :].  A copy with a gather in front: bound by the bytes of the rows read and written.  A group of
// lanes takes a row, 16 bytes of the wider type per lane and step, and several rows at a time, so that their loads are in flight together.
// 16 384 rows of 4096 from a 32-bit table of 131 072 to 16 bits: 58 us, 4.2 TB/s (a large copy: 4.76), 53 us with the same ids again; 50 021 odd rows
// of 1001: 36 us and 25.
//
// Gradient: dE[v, :] = scale * sum of the rows dout[t, :] with ids[t] = v.  Bound by the bytes of dout and dE.  Few ids make up much of a
// text, so rows of dE differ in work by orders of magnitude: the token positions are sorted by id and the sorted list is cut into chunks
// of equal length, whatever the runs in it.  A wavefront walks a chunk of a tile of columns with the sum of the current run in registers, and
// a little beyond it, to finish a run; what reaches further leaves partial rows, which a last launch adds up.  No floating-point
// atomics: the order of every sum is fixed, ascending within a chunk, in four interleaved groups over partial rows.  16 384 tokens added to
// 131 072 x 4096: sort 18, sums 66 (5.5 TB/s, with the same inputs again), partial rows 9 us; 262 144 tokens, 50 257 x 768 overwritten: 31, 131 (3.9 TB/s),
// 12 us.  What is left there: half of the second tile of columns is empty, and the tail's wavefronts store a row per token.
#include "device_util.h"
#include "vocab_util.h"

#include <algorithm>
#include <type_traits>

namespace scorch {

// ------------------------------------------------------------------------------------------
// lookup
// ------------------------------------------------------------------------------------------
struct LookupArgs {
    const int32_t *ids;
    const void *E;
    void *out;
    int64_t lde, ldo;
    int32_t tokens, vocab, d;
    int32_t lanes;  // lanes per row, a power of two
    float scale;
};

constexpr int kLookupRows = 4;  // rows a group has in flight

template <typename TE, typename TO>
__global__ __launch_bounds__(kBlock) void lookup_kernel(const LookupArgs a) {
    constexpr int N = kPer16<TE, TO>;
    const int groups = kBlock / a.lanes;
    const int group = (int)threadIdx.x / a.lanes, lane = (int)threadIdx.x % a.lanes;
    const int64_t t0 = ((int64_t)blockIdx.x * groups + group) * kLookupRows;
    const int c0 = ((int)blockIdx.y * a.lanes + lane) * N;
    if (c0 >= a.d) return;
    const int left = a.d - c0;
    const TE *src[kLookupRows];
    bool there[kLookupRows];
#pragma unroll
    for (int i = 0; i < kLookupRows; ++i) {
        const int32_t id = t0 + i < a.tokens ? a.ids[t0 + i] : -1;
        there[i] = id >= 0 && id < a.vocab;
        src[i] = static_cast<const TE *>(a.E) + (int64_t)(there[i] ? id : 0) * a.lde + c0;
    }
    float x[kLookupRows][N];
#pragma unroll
    for (int i = 0; i < kLookupRows; ++i) {
        if (!there[i]) {
#pragma unroll
            for (int j = 0; j < N; ++j) x[i][j] = 0.f;
        } else if (left >= N) {
            load_floats(src[i], x[i]);
        } else {
            load_floats_part(src[i], left, 0.f, x[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kLookupRows; ++i) {
        if (t0 + i >= a.tokens) break;
        if (there[i])
#pragma unroll
            for (int j = 0; j < N; ++j) x[i][j] *= a.scale;
        TO *dst = static_cast<TO *>(a.out) + (t0 + i) * a.ldo + c0;
        if (left >= N) store_floats(dst, x[i]);
        else store_floats_part(dst, left, x[i]);
    }
}

scorch_status_t launch_lookup(int32_t tokens, int32_t vocab, int32_t d, const int32_t *ids, const void *E, int32_t e_type, int64_t lde,
                              float scale, void *out, int32_t out_type, int64_t ldo, hipStream_t stream) {
    LookupArgs a{ids, E, out, lde, ldo, tokens, vocab, d, 1, scale};
    bool ok = true, fits = true;
    ok = with_type(e_type, [&](auto te) {
             ok = with_type(out_type, [&](auto to) {
                 typedef typename decltype(te)::type TE;
                 typedef typename decltype(to)::type TO;
                 const int64_t vectors = ((int64_t)d + kPer16<TE, TO> - 1) / kPer16<TE, TO>;
                 while (a.lanes < kBlock && a.lanes < vectors) a.lanes *= 2;
                 const int64_t rows = (int64_t)(kBlock / a.lanes) * kLookupRows;
                 const int64_t blocks = (tokens + rows - 1) / rows;
                 fits = grid_fits(blocks, kBlock);
                 if (fits)
                     hipLaunchKernelGGL((lookup_kernel<TE, TO>), dim3((uint32_t)blocks, (uint32_t)((vectors + a.lanes - 1) / a.lanes)),
                                        dim3(kBlock), 0, stream, a);
             });
         }) && ok;
    if (!ok) {
        set_error("embedding lookup: unknown type (%d, %d)", e_type, out_type);
        return SCORCH_ERR_INVALID_ARG;
    }
    if (!fits) {
        set_error("embedding lookup: %d tokens need a larger launch than HIP takes", tokens);
        return SCORCH_ERR_UNSUPPORTED;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "launch lookup_kernel");
    return SCORCH_OK;
}

// ------------------------------------------------------------------------------------------
// gradient: token positions sorted by id
// ------------------------------------------------------------------------------------------
// A stable radix sort from the lowest digit up, of digits wide enough that two passes do for a vocabulary of a million.  A pass is two
// launches: every workgroup counts the digits of its part of the list, then finds where they go from all counts and moves its part.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kDigitBits = 10;
constexpr int kBins = 1 << kDigitBits;
constexpr int kSortParts = 128;  // workgroups at most

struct SortArgs {
    const int32_t *keys_in, *perm_in;  // perm_in == nullptr: the first pass, the position itself, and keys_in are the caller's ids
    int32_t *keys_out, *perm_out;
    int32_t *counts;                   // [parts][bins]
    int32_t tokens, vocab;
    int32_t parts;
    int64_t part_len;                  // a multiple of what a workgroup takes in one step
    int32_t shift, bits;
    int32_t *long_runs;                // set to none
};

// Ids outside the table become `vocab`: sorted behind all others.
__device__ __forceinline__ int32_t sort_key(const SortArgs &a, int64_t i) {
    const int32_t k = a.keys_in[i];
    return !a.perm_in && (uint32_t)k >= (uint32_t)a.vocab ? a.vocab : k;
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs a) {
    __shared__ int32_t s_count[kBins];
    const int bins = 1 << a.bits;
    s_count[threadIdx.x] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.long_runs = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * a.part_len;
    const int64_t end = std::min<int64_t>(begin + a.part_len, a.tokens);
#pragma unroll 4
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads)
        atomicAdd(&s_count[(sort_key(a, i) >> a.shift) & (bins - 1)], 1);
    __syncthreads();
    if ((int)threadIdx.x < bins) a.counts[(int64_t)blockIdx.x * bins + threadIdx.x] = s_count[threadIdx.x];
}

// The lanes of this wavefront that hold the same digit, of those that take part.
__device__ __forceinline__ uint64_t same_digit(int digit, int bits, bool valid) {
    const uint64_t all = __ballot(valid);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        if (b >= bits) break;
        const uint32_t mine = (uint32_t)__builtin_amdgcn_sbfe(digit, b, 1);  // the bit, in all places
        const uint64_t set = __ballot(mine != 0);
        lo &= ~((uint32_t)set ^ mine);
        hi &= ~((uint32_t)(set >> 32) ^ mine);
    }
    return (uint64_t)hi << 32 | lo;
}

// Exclusive sum over the threads of a workgroup of kSortThreads.
__device__ __forceinline__ int32_t sort_scan(int32_t x, int32_t *s_wave) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int32_t sum = x;
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) {
        const int32_t y = __shfl_up(sum, o);
        if (lane >= o) sum += y;
    }
    if (lane == 63) s_wave[wv] = sum;
    __syncthreads();
    int32_t before = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) before += w < wv ? s_wave[w] : 0;
    __syncthreads();
    return before + sum - x;
}

// ROUNDS: ids per thread and step.
template <int ROUNDS>
__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(const SortArgs a) {
    extern __shared__ int32_t s_move[];  // [kSortWaves][bins]: how many of a digit, per wavefront; then where the wavefront's first goes
    __shared__ int32_t s_base[kBins];    // where the next id of a digit goes
    __shared__ int32_t s_total[kBins];
    __shared__ int32_t s_wave[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int bins = 1 << a.bits;
    int32_t *count = s_move + wv * bins;
    const int64_t begin = blockIdx.x * a.part_len;
    const int64_t end = std::min<int64_t>(begin + a.part_len, a.tokens);
    int32_t key[ROUNDS], pos[ROUNDS], place[ROUNDS];
    auto request = [&](int64_t step) {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = step + (int64_t)wv * kWave * ROUNDS + r * kWave + lane;  // a wavefront has consecutive positions
            key[r] = i < end ? sort_key(a, i) : 0;
            pos[r] = i < end && a.perm_in ? a.perm_in[i] : (int32_t)i;
        }
    };
    request(begin);  // under way while the places are worked out
    {
        // where this part's ids go: behind all of lower digits, and those of the same digit in earlier parts
        s_base[tid] = 0;
        s_total[tid] = 0;
        __syncthreads();
        const int digit = tid & (bins - 1);
        int32_t before = 0, total = 0;
#pragma unroll 8
        for (int p = tid >> a.bits; p < a.parts; p += kSortThreads >> a.bits) {
            const int32_t c = a.counts[(int64_t)p * bins + digit];
            before += p < (int)blockIdx.x ? c : 0;
            total += c;
        }
        atomicAdd(&s_base[digit], before);
        atomicAdd(&s_total[digit], total);
        __syncthreads();
        const int32_t lower = sort_scan(tid < bins ? s_total[tid] : 0, s_wave);
        if (tid < bins) s_base[tid] += lower;
    }
    for (int64_t step = begin; step < end; step += kSortThreads * ROUNDS) {
        const int64_t mine = step + (int64_t)wv * kWave * ROUNDS + lane;
        for (int i = tid; i < kSortWaves * bins; i += kSortThreads) s_move[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const bool valid = mine + r * kWave < end;
            const int digit = key[r] >> a.shift & (bins - 1);
            const uint64_t peers = same_digit(digit, a.bits, valid);
            place[r] = count[digit] + __popcll(peers & ((1ull << lane) - 1));
            wave_lds_sync();
            if (valid && (peers >> lane) == 1) count[digit] = place[r] + 1;  // the last of the peers
            wave_lds_sync();
        }
        __syncthreads();
        if (tid < bins) {
            int32_t at = s_base[tid];
            for (int w = 0; w < kSortWaves; ++w) {
                const int32_t c = s_move[w * bins + tid];
                s_move[w * bins + tid] = at;
                at += c;
            }
            s_base[tid] = at;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = mine + r * kWave;
            if (i < end) {
                const int32_t to = count[key[r] >> a.shift & (bins - 1)] + place[r];
                a.keys_out[to] = key[r];
                a.perm_out[to] = pos[r];
            }
        }
        if (end - step > kSortThreads * ROUNDS) request(step + kSortThreads * ROUNDS);
        __syncthreads();
    }
}

// For short lists: one launch, in which a workgroup has a range of ids and a part of the positions.  It reads the whole list, counts the ids of
// its range and those below it, and so knows where its own go: no workgroup waits for another.
constexpr int kRankBitsMax = kDigitBits;  // ids per range, in bits: 18 counters per id in LDS
constexpr int kRankRounds = 4;    // ids of its part that a thread holds, at most

struct RankArgs {
    const int32_t *ids;
    int32_t *keys_out, *perm_out;
    int32_t tokens, vocab;
    int32_t bits;    // of the range
    int32_t rounds;  // ids per thread of a part
    int32_t *long_runs;  // set to none
};

__global__ __launch_bounds__(kSortThreads) void rank_sort_kernel(const RankArgs a) {
    extern __shared__ int32_t s_rank[];  // [kSortWaves][range]: how many of an id the wavefront has, then where its first one goes
    __shared__ int32_t s_wave[kSortWaves];
    __shared__ int32_t s_below;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int range = 1 << a.bits;
    const int32_t lo = (int32_t)blockIdx.x << a.bits;
    int32_t *count = s_rank + wv * range;
    int32_t *s_before = s_rank + kSortWaves * range, *s_rest = s_before + range;  // in the parts before this one, and in the others
    const int32_t first = (int32_t)blockIdx.y * a.rounds * kSortThreads;          // of this part
    auto key_of = [&](int32_t id) { return (uint32_t)id >= (uint32_t)a.vocab ? a.vocab : id; };
    int32_t key[kRankRounds], place[kRankRounds];
    const int32_t mine = first + wv * kWave * a.rounds + lane;  // a wavefront has consecutive positions
#pragma unroll
    for (int r = 0; r < kRankRounds; ++r) {
        const int32_t i = mine + r * kWave;
        key[r] = r < a.rounds && i < a.tokens ? key_of(a.ids[i]) : -1;
    }
    for (int i = tid; i < (kSortWaves + 2) * range; i += kSortThreads) s_rank[i] = 0;
    if (tid == 0) s_below = 0;
    if (blockIdx.x + blockIdx.y == 0 && tid == 0) *a.long_runs = 0;
    __syncthreads();
    int32_t below = 0;
    auto look = [&](int32_t i, int32_t id) {
        const int32_t k = key_of(id);
        if (k < lo) ++below;
        else if (k - lo < range) atomicAdd(i < first ? &s_before[k - lo] : &s_rest[k - lo], 1);
    };
    constexpr int W = 4;
    int32_t i = tid * W;
#pragma unroll 2
    for (; i + W <= a.tokens; i += kSortThreads * W) {
        const typename Pack<int32_t, W>::type id = *reinterpret_cast<const typename Pack<int32_t, W>::type *>(a.ids + i);
#pragma unroll
        for (int u = 0; u < W; ++u) look(i + u, id[u]);
    }
    for (; i < a.tokens; ++i) look(i, a.ids[i]);  // the last W - 1 at most, of one thread
    for (int o = 32; o > 0; o /= 2) below += __shfl_xor(below, o);
    if (lane == 0 && below) atomicAdd(&s_below, below);
#pragma unroll
    for (int r = 0; r < kRankRounds; ++r) {
        if (r >= a.rounds) break;
        const int32_t j = key[r] - lo;
        const bool here = key[r] >= lo && j < range;  // lo >= 0
        if (__ballot(here) == 0) continue;
        const uint64_t peers = same_digit(j, a.bits, here);
        place[r] = here ? count[j] + __popcll(peers & ((1ull << lane) - 1)) : 0;
        wave_lds_sync();
        if (here && (peers >> lane) == 1) count[j] = place[r] + 1;  // the last of the peers
        wave_lds_sync();
    }
    __syncthreads();
    const int32_t before = tid < range ? s_before[tid] : 0;
    int32_t at = s_below + sort_scan(tid < range ? before + s_rest[tid] : 0, s_wave) + before;
    if (tid < range)
        for (int w = 0; w < kSortWaves; ++w) {
            const int32_t c = s_rank[w * range + tid];
            s_rank[w * range + tid] = at;
            at += c;
        }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRankRounds; ++r) {
        const int32_t j = key[r] - lo;
        if (key[r] < lo || j >= range) continue;
        const int32_t to = count[j] + place[r];
        a.keys_out[to] = key[r];
        a.perm_out[to] = mine + r * kWave;
    }
}

// ------------------------------------------------------------------------------------------
// gradient: sums of runs
// ------------------------------------------------------------------------------------------
constexpr int kFewTokens = 128;

struct RunArgs {
    const int32_t *ids;          // as they are; used instead of the sorted list of up to kFewTokens
    const int32_t *keys, *perm;  // sorted by id
    const void *dout;
    void *dE;
    float *partials;             // [chunks][2][stride]: of the run a chunk begins with, if it began before; of the run that begins in it and goes on
    int32_t *long_runs;          // how many runs have partial rows, then the chunks that they begin in
    int64_t lddo, ldde;
    int32_t tokens, vocab, d;
    int32_t chunk, chunks;       // entries per chunk
    int32_t ahead;               // entries behind its chunk that a wavefront takes to finish a run, no more than a chunk has
    int32_t tiles;               // tiles of columns
    int64_t stride;              // of the partial rows
    int64_t reduce_blocks;       // workgroups of the sums; the others store zeros
    float scale;
    int32_t fill_rows;           // rows of dE per wavefront of those
};

constexpr int kFillRowsMax = 64;  // rows of dE a wavefront looks at for ones without a token

template <typename TE, int N, bool ADD>
__device__ __forceinline__ void store_row(const RunArgs &a, int32_t id, int c0, int left, const float (&acc)[N], const typename Pack<TE, N>::type &old) {
    TE *dst = static_cast<TE *>(a.dE) + (int64_t)id * a.ldde + c0;
    float y[N];
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = ADD ? (float)old[j] + acc[j] * a.scale : acc[j] * a.scale;
    if (left >= N) store_floats(dst, y);  // streaming stores: 3 % less to 11 % more time
    else store_floats_part(dst, left, y);
}

// First place in the sorted list with an id of at least `id`.
__device__ __forceinline__ int32_t first_of(const int32_t *keys, int32_t n, int32_t id) {
    int32_t lo = 0, len = n;
    while (len > 0) {
        const int32_t half = len >> 1;
        if (keys[lo + half] < id) {
            lo += half + 1;
            len -= half + 1;
        } else {
            len = half;
        }
    }
    return lo;
}

// Rows without a token become zeros: a lane looks one id up, then the wavefront stores row by row.
template <typename TE> __device__ __forceinline__ void fill_rows(const RunArgs &a, const int32_t *keys, int64_t wave) {
    const int lane = threadIdx.x & 63;
    const int64_t v0 = wave * a.fill_rows, v = v0 + lane;
    bool empty = false;
    if (lane < a.fill_rows && v < a.vocab) {
        const int32_t p = first_of(keys, a.tokens, (int32_t)v);
        empty = p == a.tokens || keys[p] != (int32_t)v;
    }
    constexpr int M = 16 / sizeof(TE);
    const float zero[M] = {};
    for (uint64_t todo = __ballot(empty); todo; todo &= todo - 1) {
        TE *row = static_cast<TE *>(a.dE) + (v0 + __builtin_ctzll(todo)) * a.ldde;
        for (int c = lane * M; c < a.d; c += kWave * M) {
            if (a.d - c >= M) store_floats(row + c, zero);
            else store_floats_part(row + c, a.d - c, zero);
        }
    }
}

// N consecutive elements, the first `left` of them if there are fewer.
template <typename T, int N> __device__ __forceinline__ typename Pack<T, N>::type load_some(const T *p, int left) {
    typename Pack<T, N>::type v = {};
    if (left >= N) {
        v = *reinterpret_cast<const typename Pack<T, N>::type *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) v[i] = p[i];
    }
    return v;
}

// N: columns per lane.  LOADS: rows of dout in flight per wavefront.  ADD: dE holds something already; the row a run ends in is requested with
// the run's last row of dout, so that no sum waits for it.  FEW: every workgroup sorts the ids itself, which saves a launch, and every run is
// the wavefront's that it begins with, which saves another.
template <typename TD, typename TE, int N, int LOADS, bool ADD, bool FEW>
__global__ __launch_bounds__(kBlock) void run_sum_kernel(const RunArgs a) {
    __shared__ int32_t s_keys[FEW ? kFewTokens : 1], s_perm[FEW ? kFewTokens : 1], s_ids[FEW ? kFewTokens : 1];
    const int lane = threadIdx.x & 63;
    if constexpr (FEW) {
        const int tid = threadIdx.x;
        int32_t key = 0;
        if (tid < a.tokens) {
            key = a.ids[tid];
            if ((uint32_t)key >= (uint32_t)a.vocab) key = a.vocab;
            s_ids[tid] = key;
        }
        __syncthreads();
        if (tid < a.tokens) {
            int place = 0;
            for (int j = 0; j < a.tokens; ++j) place += (s_ids[j] < key) | ((s_ids[j] == key) & (j < tid));
            s_keys[place] = key;
            s_perm[place] = tid;
        }
        __syncthreads();
    }
    const int32_t *keys = FEW ? s_keys : a.keys, *perm = FEW ? s_perm : a.perm;
    if ((int64_t)blockIdx.x >= a.reduce_blocks) {
        fill_rows<TE>(a, keys, ((int64_t)blockIdx.x - a.reduce_blocks) * kWavesPerBlock + (threadIdx.x >> 6));
        return;
    }
    const int64_t unit = (int64_t)blockIdx.x * kWavesPerBlock + (threadIdx.x >> 6);
    if (unit >= (int64_t)a.chunks * a.tiles) return;
    const int64_t c = unit / a.tiles;
    const int c0 = ((int)(unit % a.tiles) * kWave + lane) * N;
    const int left = a.d - c0;  // none if it is not positive
    const int64_t begin = c * a.chunk;
    const int64_t end = std::min<int64_t>(begin + a.chunk, a.tokens), ahead = std::min<int64_t>(end + a.ahead, a.tokens);
    auto key_at = [&](int64_t i) { return i >= 0 && i < a.tokens ? keys[i] : -1; };
    const int32_t head = keys[begin], tail = keys[end - 1];
    if (head >= a.vocab) return;  // ids outside the table are the last of the list
    const bool head_earlier = key_at(begin - 1) == head;
    // A run belongs to the chunk that it begins in, if it does not reach far into the next one.
    const bool head_taken = head_earlier && (FEW || (key_at(begin - a.chunk - 1) != head && key_at(begin + a.ahead) != head));
    const bool tail_here = tail < a.vocab && key_at(end) == tail && !(head_earlier && head == tail);  // begins here and goes on
    const bool tail_whole = tail_here && (FEW || key_at(ahead) != tail);
    int64_t stop = end;
    if (tail_whole)
        for (int64_t k = end + lane;; k += kWave) {
            const uint64_t out = ~__ballot(k < ahead && keys[k] == tail);
            stop += out ? __builtin_ctzll(out) : kWave;
            if (out) break;
        }
    const TD *src = static_cast<const TD *>(a.dout) + c0;
    const TE *dst = static_cast<const TE *>(a.dE) + c0;
    float acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
    float *partial = a.partials + c * 2 * a.stride + c0;
    auto part = [&](float *p) {
        if (left >= N) store_floats(p, acc);
        else store_floats_part(p, left, acc);
    };
    bool began_here = !head_earlier;  // the current run
    for (int64_t base = begin; base < stop; base += kWave) {
        const int n = (int)std::min<int64_t>(kWave, stop - base);
        const int32_t my_key = lane < n ? keys[base + lane] : a.vocab;
        const int32_t my_next = lane < n && base + lane + 1 < a.tokens ? keys[base + lane + 1] : -1;
        const int32_t my_row = lane < n ? perm[base + lane] : 0;
        const uint64_t last = __ballot(my_key != my_next);  // of its run
        int e0 = 0;
        if (head_taken && !began_here) {
            const uint64_t others = __ballot(my_key != head);
            if (others == 0) continue;
            e0 = __builtin_ctzll(others);
            began_here = true;
        }
        for (; e0 < n; e0 += LOADS) {
            typename Pack<TD, N>::type x[LOADS];
            typename Pack<TE, N>::type old[LOADS];
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int e = std::min(e0 + u, n - 1);
                x[u] = load_some<TD, N>(src + __builtin_amdgcn_readlane(my_row, e) * a.lddo, left);
                if constexpr (ADD) {
                    const int32_t key = __builtin_amdgcn_readlane(my_key, e);
                    if (last >> e & 1 && key < a.vocab) old[u] = load_some<TE, N>(dst + key * a.ldde, left);
                }
            }
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int e = e0 + u;
                if (e >= n) break;
                const int32_t key = __builtin_amdgcn_readlane(my_key, e);
                if (key >= a.vocab) return;  // the run before them has been stored
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] += (float)x[u][j];
                if (last >> e & 1) {
                    if (left > 0) {
                        if (began_here) store_row<TE, N, ADD>(a, key, c0, left, acc, old[u]);
                        else part(partial);
                    }
                    began_here = true;
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] = 0.f;
                }
            }
        }
    }
    // a run that goes on
    if (key_at(end) != tail || tail_whole || (head_taken && head == tail)) return;
    if (left > 0) part(tail_here ? partial + a.stride : partial);
    if (!FEW && tail_here && unit % a.tiles == 0 && lane == 0) a.long_runs[1 + atomicAdd(a.long_runs, 1)] = (int32_t)c;
}

// Adds up the runs that have partial rows; the list of these runs is in any order, what is added to what is not.  A wavefront takes a run and 64 columns, 16 lanes a row, so that 32 rows are
// in flight; if the run has more, the wavefronts of the workgroup share it, in equal consecutive shares.
constexpr int kJoinThreads = 1024;
constexpr int kJoinWaves = kJoinThreads / kWave;
constexpr int kJoinLanes = 16;
constexpr int kJoinColumns = 4 * kJoinLanes;
constexpr int kJoinGroups = kWave / kJoinLanes;
constexpr int kJoinLoads = 8;
constexpr int kJoinShort = kJoinGroups * kJoinLoads;  // partial rows that are one wavefront's

template <typename TE, bool ADD>
__global__ __launch_bounds__(kJoinThreads) void run_join_kernel(const RunArgs a) {
    constexpr int N = 4;
    __shared__ float s_acc[kJoinWaves][kJoinLanes][N];
    __shared__ int64_t s_rows[kJoinWaves];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int col = lane % kJoinLanes, group = lane / kJoinLanes;
    const int c0 = (int)blockIdx.y * kJoinColumns + col * N;
    const int left = a.d - c0;
    // partial rows k in [from, to) of the run that begins in chunk c: the end of c, then the beginnings of c + 1, ...; the sum in all groups
    auto add = [&](int64_t c, int64_t from, int64_t to, float (&acc)[N]) {
        if (left > 0)
            for (int64_t k0 = from; k0 < to; k0 += kJoinShort) {
                float x[kJoinLoads][N];
#pragma unroll
                for (int u = 0; u < kJoinLoads; ++u) {
                    const int64_t k = std::min(k0 + u * kJoinGroups + group, to - 1);
                    load_floats(a.partials + ((c + k) * 2 + (k == 0)) * a.stride + c0, x[u]);  // rows of partials are padded
                }
#pragma unroll
                for (int u = 0; u < kJoinLoads; ++u)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] += k0 + u * kJoinGroups + group < to ? x[u][j] : 0.f;
            }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            acc[j] += lane_xor<16>(acc[j]);
            acc[j] += lane_xor<32>(acc[j]);
        }
    };
    auto held = [&](int32_t id) {  // requested before the partial rows
        return ADD ? load_some<TE, N>(static_cast<const TE *>(a.dE) + id * a.ldde + c0, left) : typename Pack<TE, N>::type{};
    };
    const int32_t n_runs = a.long_runs[0];
    // neighbours in the list, often long runs next to each other, go to different workgroups
    for (int32_t first = (int32_t)blockIdx.x; first < n_runs; first += (int32_t)gridDim.x * kJoinWaves) {
        int64_t rows = 0;
        const int64_t mine = first + (int64_t)wv * gridDim.x;
        if (mine < n_runs) {
            const int64_t c = a.long_runs[1 + mine];
            const int32_t id = a.keys[(c + 1) * a.chunk];
            // the chunks behind c that begin with the run: all up to the last whose first id it is
            for (rows = 2;; rows += kWave) {
                const int64_t k = c + rows + lane;
                const uint64_t out = ~__ballot(k < a.chunks && a.keys[k * a.chunk] == id);
                if (out) {
                    rows += __builtin_ctzll(out);
                    break;
                }
            }
            if (rows <= kJoinShort) {
                float acc[N] = {};
                const auto old = held(id);
                add(c, 0, rows, acc);
                if (left > 0 && group == 0) store_row<TE, N, ADD>(a, id, c0, left, acc, old);
                rows = 0;
            }
        }
        if (lane == 0) s_rows[wv] = rows;
        __syncthreads();
        for (int w = 0; w < kJoinWaves; ++w) {
            const int64_t n = s_rows[w];
            if (n == 0) continue;
            const int64_t c = a.long_runs[1 + first + (int64_t)w * gridDim.x];
            const int32_t id = a.keys[(c + 1) * a.chunk];
            float acc[N] = {};
            typename Pack<TE, N>::type old = {};
            if (wv == 0) old = held(id);
            add(c, n * wv / kJoinWaves, n * (wv + 1) / kJoinWaves, acc);
            if (group == 0)
#pragma unroll
                for (int j = 0; j < N; ++j) s_acc[wv][col][j] = acc[j];
            __syncthreads();
            if (wv == 0) {
                for (int o = 1; o < kJoinWaves; ++o)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] += s_acc[o][col][j];
                if (left > 0 && group == 0) store_row<TE, N, ADD>(a, id, c0, left, acc, old);
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

struct GradLayout {
    uint64_t off_keys[2], off_perm[2], off_counts, off_long, off_partials, total;
    int32_t chunk, chunks;
    int64_t stride;
};

// Entries per chunk: as many as leave 4096 wavefronts (16 per CU), counted in tiles of 512 columns, between 8 and 256.
static GradLayout layout_gradient(int32_t tokens, int32_t d) {
    GradLayout l{};
    const int64_t tiles = std::max<int64_t>(1, ((int64_t)d + 511) / 512);
    l.chunk = 8;
    while (l.chunk < 256 && (int64_t)tokens * tiles / l.chunk >= 2 * 4096) l.chunk *= 2;
    l.chunks = (int32_t)(((int64_t)tokens + l.chunk - 1) / l.chunk);
    l.stride = ((int64_t)d + 63) / 64 * 64;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        l.off_keys[i] = take((uint64_t)tokens * 4);
        l.off_perm[i] = take((uint64_t)tokens * 4);
    }
    l.off_counts = take((uint64_t)kSortParts * kBins * 4);
    l.off_long = take(((uint64_t)l.chunks + 1) * 4);
    l.off_partials = take((uint64_t)l.chunks * 2 * l.stride * 4);
    l.total = at;
    return l;
}

uint64_t gradient_workspace_bytes(int32_t tokens, int32_t d) { return layout_gradient(tokens, d).total; }

// The one-launch sort reads the list once per range of ids and part, so it is for as many workgroups as run at once (two per CU) and not too long
// lists.  Measured, one launch / radix passes: vocabulary 32 000, 256 tokens 4.4 / 11 us, 2048 4.9 / 14, 8192 7.2 / 15, 16 384 9.5 / 16, 32 768
// 14.5 / 16.6, 65 536 29 / 17; 131 072, 2048 6.8 / 14.5, 8192 10.4 / 18, 16 384 16.1 / 17.3, 32 768 29 / 19; 262 144, 2048 7.7 / 16, 8192 14.9 / 18,
// 16 384 22 / 19.  Ranges of more ids before parts of more: 32 000 and 8192, 32 ranges x 8 parts 7.2, 126 x 2 8.8, 126 x 8 12.
constexpr int32_t kRankTokensMax = 32768;
constexpr int64_t kRankGroups = kCus + 8;  // ranges x parts: the range that holds the key of ids outside the table may be one more

// The token positions in the order of their ids, and of themselves where these are equal; ids outside the table count as vocab.
static void sort_by_id(int32_t tokens, int32_t vocab, const int32_t *ids, char *workspace, const GradLayout &l, hipStream_t stream,
                       const int32_t *&keys, const int32_t *&perm) {
    if (tokens == 0) return;
    int32_t *keys_out[2], *perm_out[2];
    for (int i = 0; i < 2; ++i) {
        keys_out[i] = reinterpret_cast<int32_t *>(workspace + l.off_keys[i]);
        perm_out[i] = reinterpret_cast<int32_t *>(workspace + l.off_perm[i]);
    }
    int32_t *long_runs = reinterpret_cast<int32_t *>(workspace + l.off_long);
    RankArgs k{ids, keys_out[0], perm_out[0], tokens, vocab, 6, 1, long_runs};
    auto ranges = [&] { return ((int64_t)vocab >> k.bits) + 1; };  // of the ids 0 ... vocab
    auto parts = [&] { return ((int64_t)tokens + k.rounds * kSortThreads - 1) / (k.rounds * kSortThreads); };
    while (k.bits < kRankBitsMax && ranges() * parts() > kRankGroups) ++k.bits;
    while (k.rounds < kRankRounds && ranges() * parts() > kRankGroups) k.rounds *= 2;
    if (tokens <= kRankTokensMax && ranges() * parts() <= 2 * kRankGroups) {
        hipLaunchKernelGGL(rank_sort_kernel, dim3((uint32_t)ranges(), (uint32_t)parts()), dim3(kSortThreads),
                           (uint32_t)((kSortWaves + 2) << k.bits) * 4, stream, k);
        keys = k.keys_out;
        perm = k.perm_out;
        return;
    }
    SortArgs s{};
    s.tokens = tokens;
    s.vocab = vocab;
    s.counts = reinterpret_cast<int32_t *>(workspace + l.off_counts);
    s.long_runs = long_runs;
    s.keys_in = ids;
    const int key_bits = 32 - __builtin_clz((uint32_t)vocab);  // ids go up to vocab itself; vocab > 0
    const int passes = (key_bits + kDigitBits - 1) / kDigitBits;
    int rounds = 1;
    while (rounds < 8 && (int64_t)tokens > (int64_t)kSortParts * kSortThreads * rounds) rounds *= 2;
    const int64_t step = kSortThreads * rounds;
    const int64_t steps = ((int64_t)tokens + step - 1) / step;
    s.part_len = (steps + kSortParts - 1) / kSortParts * step;
    s.parts = (int32_t)((tokens + s.part_len - 1) / s.part_len);
    const auto move = rounds == 1 ? sort_move_kernel<1> : rounds == 2 ? sort_move_kernel<2> : rounds == 4 ? sort_move_kernel<4> : sort_move_kernel<8>;
    for (int p = 0; p < passes; ++p) {
        s.shift = key_bits * p / passes;
        s.bits = key_bits * (p + 1) / passes - s.shift;
        s.keys_out = keys_out[p & 1];
        s.perm_out = perm_out[p & 1];
        hipLaunchKernelGGL(sort_count_kernel, dim3((uint32_t)s.parts), dim3(kSortThreads), 0, stream, s);
        hipLaunchKernelGGL(move, dim3((uint32_t)s.parts), dim3(kSortThreads), (uint32_t)(kSortWaves << s.bits) * 4, stream, s);
        s.keys_in = s.keys_out;
        s.perm_in = s.perm_out;
    }
    keys = s.keys_in;
    perm = s.perm_in;
}

scorch_status_t launch_gradient(int32_t tokens, int32_t vocab, int32_t d, const int32_t *ids, const void *dout, int32_t dout_type,
                                int64_t lddo, float scale, int32_t accumulate, void *dE, int32_t de_type, int64_t ldde,
                                char *workspace, hipStream_t stream) {
    const GradLayout l = layout_gradient(tokens, d);
    RunArgs r{};
    int64_t fill = 0;  // workgroups that store zeros: some 8192 wavefronts, more for the largest tables
    if (!accumulate) {
        r.fill_rows = 4;
        while (r.fill_rows < kFillRowsMax && vocab / r.fill_rows > 8192) r.fill_rows *= 2;
        fill = ((int64_t)vocab + r.fill_rows * kWavesPerBlock - 1) / (r.fill_rows * kWavesPerBlock);
    }
    const int64_t tiles = ((int64_t)d + kWave * 4 - 1) / (kWave * 4);  // of 32 bits, the more
    if (!grid_fits(l.chunks * tiles / kWavesPerBlock + 1 + fill, kBlock)) {
        set_error("embedding gradient: %d tokens, %d ids and %d columns need a larger launch than HIP takes", tokens, vocab, d);
        return SCORCH_ERR_UNSUPPORTED;
    }
    const bool few = tokens <= kFewTokens;
    const int32_t *keys = nullptr, *perm = nullptr;
    if (!few) sort_by_id(tokens, vocab, ids, workspace, l, stream, keys, perm);
    r.keys = keys;
    r.perm = perm;
    r.dout = dout;
    r.dE = dE;
    r.partials = reinterpret_cast<float *>(workspace + l.off_partials);
    r.long_runs = reinterpret_cast<int32_t *>(workspace + l.off_long);
    r.lddo = lddo;
    r.ldde = ldde;
    r.tokens = tokens;
    r.vocab = vocab;
    r.d = d;
    r.chunk = l.chunk;
    r.chunks = l.chunks;
    r.ahead = few ? tokens : std::max(8, l.chunk / 4);
    r.ids = ids;
    r.stride = l.stride;
    r.scale = scale;
    bool ok = true;
    ok = with_type(dout_type, [&](auto td) {
             ok = with_type(de_type, [&](auto te) {
                 typedef typename decltype(td)::type TD;
                 typedef typename decltype(te)::type TE;
                 constexpr int N = 16 / sizeof(TD);
                 r.tiles = (d + kWave * N - 1) / (kWave * N);
                 r.reduce_blocks = ((int64_t)r.chunks * r.tiles + kWavesPerBlock - 1) / kWavesPerBlock;
                 const int32_t column_tiles = (d + kJoinColumns - 1) / kJoinColumns;
                 const dim3 sums((uint32_t)(r.reduce_blocks + fill)), joins((uint32_t)std::max(1, std::min((r.chunks + kJoinWaves - 1) / kJoinWaves, 2 * kCus / column_tiles)), (uint32_t)column_tiles);
                 auto launch = [&](auto add) {
                     constexpr bool ADD = decltype(add)::value;
                     constexpr int LOADS = ADD ? 4 : 8;
                     if (sums.x == 0) return;
                     if (few) hipLaunchKernelGGL((run_sum_kernel<TD, TE, N, LOADS, ADD, true>), sums, dim3(kBlock), 0, stream, r);
                     else hipLaunchKernelGGL((run_sum_kernel<TD, TE, N, LOADS, ADD, false>), sums, dim3(kBlock), 0, stream, r);
                     if (!few && r.chunks > 1) hipLaunchKernelGGL((run_join_kernel<TE, ADD>), joins, dim3(kJoinThreads), 0, stream, r);
                 };
                 if (accumulate) launch(std::true_type());
                 else launch(std::false_type());
             });
         }) && ok;
    if (!ok) {
        set_error("embedding gradient: unknown type (%d, %d)", dout_type, de_type);
        return SCORCH_ERR_INVALID_ARG;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "launch of the embedding gradient");
    return SCORCH_OK;
}

}  // namespace scorch
