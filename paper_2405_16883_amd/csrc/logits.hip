// Logits of the next token before it is chosen: penalties for tokens of the history, biases and grammar masks (definition in
// scorch_spmm.h).
//
// Bound by the bytes of the logits read and written.  A workgroup has a tile of columns of one row, for which it counts in LDS how often
// each token occurs in the row's history, with the tile's logits already on their way to registers.  Counts are whole numbers, so the
// order of the atomic additions changes nothing.  Biases are looked up in LDS too; where a column has several, its first entry adds them up in
// the order of the list.
#include "device_util.h"
#include "vocab_util.h"

#include <algorithm>
#include <type_traits>

namespace scorch {

constexpr int kLogitsThreads = 1024;
constexpr int kLogitsVectors = 2;       // vectors of logits a thread holds
constexpr int kHistoryLoads = 4;        // tokens of the history a thread has in flight
constexpr uint32_t kSeen = 1u << 31;    // beside the count: the token occurs before generated_from

struct LogitsArgs {
    const void *in;
    void *out;
    scorch_logits_rules_t rules;
    int64_t ldi, ldo;
    int32_t rows, vocab;
    int32_t tile, tiles;  // columns per workgroup, a multiple of 32
};

// A workgroup's lists in LDS.  HISTORY: a word per column, how often from generated_from on, and kSeen.  BIAS: the value per column, a bit per
// column with entries, a bit per column with several, and the row's first entries as they are.
template <bool HISTORY, bool BIAS> struct LogitsLds {
    static constexpr int kEntries = kLogitsThreads;
    uint32_t *count, *biased, *twice;
    float *bias;
    int2 *entries;
    __device__ __forceinline__ LogitsLds(uint32_t *s, int tile) {
        count = s;
        bias = reinterpret_cast<float *>(s + (HISTORY ? tile : 0));
        biased = reinterpret_cast<uint32_t *>(bias + tile);
        twice = biased + tile / 32;
        entries = reinterpret_cast<int2 *>(twice + tile / 32);
    }
    static uint32_t bytes(int tile) { return (uint32_t)tile * 4 * HISTORY + ((uint32_t)tile * 4 + (uint32_t)tile / 16 * 4 + kEntries * 8) * BIAS; }
};

template <typename TI, typename TO, bool HISTORY, bool BIAS>
__global__ __launch_bounds__(kLogitsThreads, 8) void logits_kernel(const LogitsArgs a) {
    constexpr int N = kPer16<TI, TO>;
    extern __shared__ __attribute__((aligned(16))) uint32_t s_lds[];
    __shared__ int32_t s_several;  // some column of the tile has several bias entries
    const LogitsLds<HISTORY, BIAS> s(s_lds, a.tile);
    const scorch_logits_rules_t &r = a.rules;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x / a.tiles;
    // consecutive workgroups are on different XCDs: the tiles of the next row begin one further, or those with the most frequent tokens
    // would all be on one
    const int32_t lo = (int32_t)((blockIdx.x + row) % a.tiles) * a.tile;
    const int32_t cols = std::min(a.tile, a.vocab - lo);
    // what will be needed is requested at once: the logits, the mask and the beginnings of the lists
    float x[kLogitsVectors][N];
    uint32_t allowed[kLogitsVectors];
    {
        const TI *in = static_cast<const TI *>(a.in) + row * a.ldi + lo;
        const uint32_t *mask = r.mask ? r.mask + row * r.ldm + lo / 32 : nullptr;
#pragma unroll
        for (int u = 0; u < kLogitsVectors; ++u) {
            const int j = (u * kLogitsThreads + tid) * N;
            allowed[u] = ~0u;
            if (j >= cols) continue;
            if (cols - j >= N) load_floats(in + j, x[u]);
            else load_floats_part(in + j, cols - j, 0.f, x[u]);
            if (mask) allowed[u] = mask[j >> 5] >> (j & 31);
        }
    }
    const int32_t h0 = HISTORY ? r.history_rowptr[row] : 0, nh = HISTORY ? r.history_rowptr[row + 1] - h0 : 0;
    const int32_t b0 = BIAS ? r.bias_rowptr[row] : 0, nb = BIAS ? r.bias_rowptr[row + 1] - b0 : 0;
    int32_t token[kHistoryLoads];
    auto request = [&](int32_t q) {
#pragma unroll
        for (int u = 0; u < kHistoryLoads; ++u) {
            const int64_t p = (int64_t)q + u * kLogitsThreads;
            token[u] = p < nh ? r.history[h0 + p] : -1;
        }
    };
    if constexpr (HISTORY) request(tid);
    int32_t b_token = -1;
    float b_value = 0.f;
    if (BIAS && tid < nb) {
        b_token = r.bias_tokens[b0 + tid];
        b_value = r.bias_vals[b0 + tid];
    }
    if constexpr (HISTORY)
        for (int i = tid * 4; i < a.tile; i += kLogitsThreads * 4) *reinterpret_cast<int4 *>(s.count + i) = int4{0, 0, 0, 0};
    if constexpr (BIAS) {
        for (int i = tid; i < a.tile / 16; i += kLogitsThreads) s.biased[i] = 0;  // and twice, which follows
        s.entries[tid] = int2{b_token, __float_as_int(b_value)};
        if (tid == 0) s_several = 0;
    }
    if constexpr (HISTORY || BIAS) __syncthreads();
    if constexpr (HISTORY) {
        const int32_t from = r.generated_from ? r.generated_from[row] : 0;
        for (int32_t q = tid;;) {
#pragma unroll
            for (int u = 0; u < kHistoryLoads; ++u) {
                const int32_t j = token[u] - lo;
                const bool here = token[u] >= lo && j < cols;  // lo >= 0
                const bool counts = q + u * kLogitsThreads >= from;
                if (here && !counts) atomicOr(&s.count[j], kSeen);
                if (here && counts) atomicAdd(&s.count[j], 1u);
            }
            if (nh - q <= kHistoryLoads * kLogitsThreads) break;
            q += kHistoryLoads * kLogitsThreads;
            request(q);
        }
    }
    bool claimed = false;  // this thread's first entry is the one that found its column without any
    if constexpr (BIAS) {
        for (int32_t p = tid;;) {
            const int32_t j = b_token - lo;
            if (b_token >= lo && j < cols) {
                const uint32_t bit = 1u << (j & 31);
                if (atomicOr(&s.biased[j >> 5], bit) & bit) {
                    atomicOr(&s.twice[j >> 5], bit);
                    s_several = 1;
                } else {
                    s.bias[j] = b_value;
                    claimed = true;
                }
            }
            if (nb - p <= kLogitsThreads) break;
            p += kLogitsThreads;
            b_token = r.bias_tokens[b0 + p];
            b_value = r.bias_vals[b0 + p];
        }
    }
    if constexpr (HISTORY || BIAS) __syncthreads();
    if (BIAS && s_several) {
        // columns with several entries: these are added up in the order of the list
        if (nb <= kLogitsThreads) {
            // by the wavefront of the entry that came first, which looks at 64 entries at a time
            const int32_t at = b_token - lo;
            const bool mine = claimed && (s.twice[at >> 5] >> (at & 31) & 1);
            for (uint64_t todo = __ballot(mine); todo; todo &= todo - 1) {
                const int32_t t = __builtin_amdgcn_readlane(b_token, __builtin_ctzll(todo));
                float sum = 0.f;
                for (int32_t o = 0; o < nb; o += kWave) {
                    const int2 e = s.entries[o + lane];  // behind the last: -1, which is no token
                    for (uint64_t same = __ballot(e.x == t); same; same &= same - 1)
                        sum += __int_as_float(__builtin_amdgcn_readlane(e.y, __builtin_ctzll(same)));
                }
                if (lane == 0) s.bias[t - lo] = sum;
            }
        } else {
            // by the thread of the first entry in the list
            for (int32_t p = tid; p < nb; p += kLogitsThreads) {
                const int32_t t = r.bias_tokens[b0 + p], j = t - lo;
                if (t < lo || j >= cols || !(s.twice[j >> 5] >> (j & 31) & 1)) continue;
                bool first = true;
                float sum = 0.f;
#pragma unroll 8
                for (int32_t o = 0; o < nb; ++o) {
                    const int32_t other = r.bias_tokens[b0 + o];
                    const float value = r.bias_vals[b0 + o];
                    first &= (other != t) | (o >= p);
                    sum += other == t ? value : 0.f;
                }
                if (first) s.bias[j] = sum;
            }
        }
        __syncthreads();
    }
    TO *out = static_cast<TO *>(a.out) + row * a.ldo + lo;
    const bool repeats = HISTORY && r.repetition;
    const float repetition = repeats ? r.repetition[row] : 1.f;
    const float frequency = HISTORY && r.frequency ? r.frequency[row] : 0.f, presence = HISTORY && r.presence ? r.presence[row] : 0.f;
#pragma unroll
    for (int u = 0; u < kLogitsVectors; ++u) {
        const int j = (u * kLogitsThreads + tid) * N;
        if (j >= cols) continue;
        if constexpr (HISTORY)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t c = s.count[j + i];  // 0 behind the last column
                if (c == 0) continue;
                if (repeats) x[u][i] = x[u][i] > 0.f ? x[u][i] / repetition : x[u][i] * repetition;
                const uint32_t times = c & ~kSeen;
                if (times) x[u][i] = x[u][i] - frequency * (float)times - presence;
            }
        if constexpr (BIAS)
            for (uint32_t b = s.biased[j >> 5] >> (j & 31) & ((1u << N) - 1); b; b &= b - 1) {
                const int at = __builtin_ctz(b);
                const float v = s.bias[j + at];
#pragma unroll
                for (int i = 0; i < N; ++i) x[u][i] += i == at ? v : 0.f;
            }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(allowed[u] >> i & 1)) x[u][i] = -INFINITY;
        if (cols - j >= N) store_floats(out + j, x[u]);
        else store_floats_part(out + j, cols - j, x[u]);
    }
}

scorch_status_t launch_logits(int32_t rows, int32_t vocab, const void *in, int32_t type, int64_t ldi, const scorch_logits_rules_t &rules,
                              void *out, int32_t out_type, int64_t ldo, hipStream_t stream) {
    LogitsArgs a{in, out, rules, ldi, ldo, rows, vocab, 0, 0};
    a.tile = kLogitsThreads * kLogitsVectors * (type == SCORCH_TYPE_F32 || out_type == SCORCH_TYPE_F32 ? 4 : 8);  // kPer16 of the types
    a.tiles = (vocab + a.tile - 1) / a.tile;
    const int64_t grid = (int64_t)rows * a.tiles;
    if (!grid_fits(grid, kLogitsThreads)) {
        set_error("logits: %d rows of %d columns need a larger launch than HIP takes", rows, vocab);
        return SCORCH_ERR_UNSUPPORTED;
    }
    bool ok = true;
    ok = with_type(type, [&](auto ti) {
             ok = with_type(out_type, [&](auto to) {
                 typedef typename decltype(ti)::type TI;
                 typedef typename decltype(to)::type TO;
                 auto launch = [&](auto history, auto bias) {
                     constexpr bool H = decltype(history)::value, B = decltype(bias)::value;
                     hipLaunchKernelGGL((logits_kernel<TI, TO, H, B>), dim3((uint32_t)grid), dim3(kLogitsThreads),
                                        (LogitsLds<H, B>::bytes(a.tile)), stream, a);
                 };
                 typedef std::true_type yes;
                 typedef std::false_type no;
                 if (rules.history_rowptr && rules.bias_rowptr) launch(yes(), yes());
                 else if (rules.history_rowptr) launch(yes(), no());
                 else if (rules.bias_rowptr) launch(no(), yes());
                 else launch(no(), no());
             });
         }) && ok;
    if (!ok) {
        set_error("logits: unknown type (%d, %d)", type, out_type);
        return SCORCH_ERR_INVALID_ARG;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "launch logits_kernel");
    return SCORCH_OK;
}

}  // namespace scorch
