// Logits of the next token before it is chosen: penalties for tokens of the history, biases and grammar masks (definition in
// scorch_spmm.h).
//
// Bound by the bytes of the logits read and written.  A workgroup has some tiles of columns of one row.  For a tile it counts in LDS how often
// each token occurs in the row's history and looks the biases up there, with the tile's logits already on their way to registers; then it passes
// over the tile once.  Counts are whole numbers, so the order of the atomic additions changes nothing.  Where a column has several biases, they are
// added up in the order of the list.  256 rows of 131 072, bf16 to f32, histories of 2048, 64 biases, mask: 43 us, 57 when nothing is in a cache (a
// plain copy 29 and 43); without biases 35.  33 rows of 50 257 with histories of 32 768 and 300 biases: 21 us, of which 8 go into biases
// that repeat a token and 4 into the history, both on the one CU that has the row's most frequent tokens; with distinct biases 12.5.
// From 16 to 16 bits a vector has 8 columns and a tile 16 384: LDS has room for one workgroup per CU if there are biases (80 KB, 144 KB with a history),
// and the same batch takes 46 us where a copy takes 20.  64 registers, for two workgroups per CU, are up to 10 too few; no form without spills was measured.
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
    int32_t tile, tiles;  // columns worked on at a time, a multiple of 32
    int32_t parts;        // workgroups per row
};

// A workgroup's lists in LDS.  HISTORY: a word per column, how often from generated_from on, and kSeen.  BIAS: the value per column, a bit per
// column with entries and a bit per column with several (for the tile at hand and the next), and the row's first entries as they are.
template <bool HISTORY, bool BIAS> struct LogitsLds {
    static constexpr int kEntries = kLogitsThreads;
    uint32_t *count, *marks;
    float *bias;
    int2 *entries;
    __device__ __forceinline__ LogitsLds(uint32_t *s, int tile) {
        count = s;
        bias = reinterpret_cast<float *>(s + (HISTORY ? tile : 0));
        marks = reinterpret_cast<uint32_t *>(bias + tile);  // [2][biased, twice][tile / 32]
        entries = reinterpret_cast<int2 *>(marks + tile / 8);
    }
    static uint32_t bytes(int tile) { return (uint32_t)tile * 4 * HISTORY + ((uint32_t)tile * 4 + (uint32_t)tile / 8 * 4 + kEntries * 8) * BIAS; }
};

// A workgroup has every `parts`-th tile of a row.  While it works on one, the logits of its next are on their way; the lists are read once, as far
// as they fit into registers.
template <typename TI, typename TO, bool HISTORY, bool BIAS>
__global__ __launch_bounds__(kLogitsThreads, 8) void logits_kernel(const LogitsArgs a) {
    constexpr int N = kPer16<TI, TO>;
    extern __shared__ __attribute__((aligned(16))) uint32_t s_lds[];
    __shared__ int32_t s_several[2];  // some column of the tile has several bias entries
    const LogitsLds<HISTORY, BIAS> s(s_lds, a.tile);
    const scorch_logits_rules_t &r = a.rules;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x / a.parts;
    // Consecutive workgroups are on different XCDs: the parts of the next row begin one further, or those with the most frequent tokens would all
    // be on one.
    const int32_t part = (int32_t)((blockIdx.x + row) % a.parts);
    const TI *in = static_cast<const TI *>(a.in) + row * a.ldi;
    TO *out = static_cast<TO *>(a.out) + row * a.ldo;
    const uint32_t *mask = r.mask ? r.mask + row * r.ldm : nullptr;
    raw16 now[kLogitsVectors], next[kLogitsVectors];  // as they are in memory: fewer registers
    uint32_t allowed[kLogitsVectors], allowed_next[kLogitsVectors];
    auto request = [&](int32_t lo) {
        const int32_t cols = std::min(a.tile, a.vocab - lo);
#pragma unroll
        for (int u = 0; u < kLogitsVectors; ++u) {
            const int j = (u * kLogitsThreads + tid) * N;
            allowed_next[u] = ~0u;
            if (j >= cols) continue;
            if (cols - j >= N) next[u] = load_raw<TI, N * sizeof(TI)>(in + lo + j);
            if (mask) allowed_next[u] = mask[(lo + j) >> 5] >> (j & 31);
        }
    };
    request(part * a.tile);
    const int32_t h0 = HISTORY ? r.history_rowptr[row] : 0, nh = HISTORY ? r.history_rowptr[row + 1] - h0 : 0;
    const int32_t b0 = BIAS ? r.bias_rowptr[row] : 0, nb = BIAS ? r.bias_rowptr[row + 1] - b0 : 0;
    int32_t token[kHistoryLoads];
    auto request_tokens = [&](int32_t q) {
#pragma unroll
        for (int u = 0; u < kHistoryLoads; ++u) {
            const int64_t p = (int64_t)q + u * kLogitsThreads;
            token[u] = p < nh ? r.history[h0 + p] : -1;
        }
    };
    if constexpr (HISTORY) request_tokens(tid);

    int32_t first_token = -1;
    float first_value = 0.f;
    if (BIAS && tid < nb) {
        first_token = r.bias_tokens[b0 + tid];
        first_value = r.bias_vals[b0 + tid];
    }
    const int32_t from = HISTORY && r.generated_from ? r.generated_from[row] : 0;
    const bool repeats = HISTORY && r.repetition;
    const float repetition = repeats ? r.repetition[row] : 1.f;
    const float frequency = HISTORY && r.frequency ? r.frequency[row] : 0.f, presence = HISTORY && r.presence ? r.presence[row] : 0.f;
    if constexpr (HISTORY)
        for (int i = tid * 4; i < a.tile; i += kLogitsThreads * 4) *reinterpret_cast<int4 *>(s.count + i) = int4{0, 0, 0, 0};
    if constexpr (BIAS) {
        for (int i = tid; i < a.tile / 8; i += kLogitsThreads) s.marks[i] = 0;
        s.entries[tid] = int2{first_token, __float_as_int(first_value)};
        if (tid < 2) s_several[tid] = 0;
    }
    if constexpr (HISTORY || BIAS) __syncthreads();
    int which = 0;
    for (int32_t t = part; t < a.tiles; t += a.parts) {
        const int32_t lo = t * a.tile;
        const int32_t cols = std::min(a.tile, a.vocab - lo);
#pragma unroll
        for (int u = 0; u < kLogitsVectors; ++u) {
            allowed[u] = allowed_next[u];
            now[u] = next[u];
        }
        if (a.tiles - t > a.parts) request(lo + a.parts * a.tile);
        uint32_t *s_biased = s.marks + which * (a.tile / 16), *s_twice = s_biased + a.tile / 32;
        if constexpr (HISTORY) {
            for (int32_t q = tid;;) {
#pragma unroll
                for (int u = 0; u < kHistoryLoads; ++u) {
                    const int32_t j = token[u] - lo;
                    if (token[u] < lo || j >= cols) continue;  // lo >= 0
                    if (q + u * kLogitsThreads >= from) atomicAdd(&s.count[j], 1u);
                    else atomicOr(&s.count[j], kSeen);
                }
                if (nh - q <= kHistoryLoads * kLogitsThreads) break;
                q += kHistoryLoads * kLogitsThreads;
                request_tokens(q);
            }
            if (nh > kHistoryLoads * kLogitsThreads) request_tokens(tid);  // for the next tile
        }
        bool claimed = false;  // this thread's first entry is the one that found its column without any
        if constexpr (BIAS) {
            int32_t token = first_token;
            float value = first_value;
            for (int32_t p = tid;;) {
                const int32_t j = token - lo;
                if (token >= lo && j < cols) {
                    const uint32_t bit = 1u << (j & 31);
                    if (atomicOr(&s_biased[j >> 5], bit) & bit) {
                        atomicOr(&s_twice[j >> 5], bit);
                        s_several[which] = 1;
                    } else {
                        s.bias[j] = value;
                        claimed = p == tid;
                    }
                }
                if (nb - p <= kLogitsThreads) break;
                p += kLogitsThreads;
                token = r.bias_tokens[b0 + p];
                value = r.bias_vals[b0 + p];
            }
        }
        if constexpr (HISTORY || BIAS) __syncthreads();
        if (BIAS && s_several[which]) {
            // columns with several entries: these are added up in the order of the list
            if (nb <= kLogitsThreads) {
                // by the wavefront of the entry that came first, which looks at 64 entries at a time
                const int32_t at = first_token - lo;
                const bool mine = claimed && (s_twice[at >> 5] >> (at & 31) & 1);
                for (uint64_t todo = __ballot(mine); todo; todo &= todo - 1) {
                    const int32_t token = __builtin_amdgcn_readlane(first_token, __builtin_ctzll(todo));
                    float sum = 0.f;
                    for (int32_t o = 0; o < nb; o += kWave) {
                        const int2 e = s.entries[o + lane];  // behind the last: -1, which is no token
                        for (uint64_t same = __ballot(e.x == token); same; same &= same - 1)
                            sum += __int_as_float(__builtin_amdgcn_readlane(e.y, __builtin_ctzll(same)));
                    }
                    if (lane == 0) s.bias[token - lo] = sum;
                }
            } else {
                // by the thread of the first entry in the list
                for (int32_t p = tid; p < nb; p += kLogitsThreads) {
                    const int32_t token = r.bias_tokens[b0 + p], j = token - lo;
                    if (token < lo || j >= cols || !(s_twice[j >> 5] >> (j & 31) & 1)) continue;
                    bool first = true;
                    float sum = 0.f;
#pragma unroll 2
                    for (int32_t o = 0; o < nb; ++o) {
                        const int32_t other = r.bias_tokens[b0 + o];
                        const float value = r.bias_vals[b0 + o];
                        first &= (other != token) | (o >= p);
                        sum += other == token ? value : 0.f;
                    }
                    if (first) s.bias[j] = sum;
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kLogitsVectors; ++u) {
            const int j = (u * kLogitsThreads + tid) * N;
            if (j >= cols) continue;
            float x[N];
            if (cols - j >= N) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = element<TI>(now[u], i);
            } else {
                load_floats_part(in + lo + j, cols - j, 0.f, x);
            }
            if constexpr (HISTORY) {
                typedef uint32_t counts __attribute__((ext_vector_type(4)));
#pragma unroll
                for (int h = 0; h < N / 4; ++h) {
                    counts *at = reinterpret_cast<counts *>(s.count + j + 4 * h);  // 0 behind the last column
                    const counts c = *at;
                    if ((c[0] | c[1] | c[2] | c[3]) == 0) continue;
                    *at = counts{0, 0, 0, 0};  // for the next tile
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float y = x[4 * h + i];
                        if (repeats && c[i] != 0) y = y > 0.f ? y / repetition : y * repetition;
                        const uint32_t times = c[i] & ~kSeen;
                        x[4 * h + i] = times ? y - frequency * (float)times - presence : y;
                    }
                }
            }
            if constexpr (BIAS)
                for (uint32_t b = s_biased[j >> 5] >> (j & 31) & ((1u << N) - 1); b; b &= b - 1) {
                    const int at = __builtin_ctz(b);
                    const float v = s.bias[j + at];
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] = i == at ? x[i] + v : x[i];  // the others keep their bits
                }
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(allowed[u] >> i & 1)) x[i] = -INFINITY;
            if (cols - j >= N) store_floats(out + lo + j, x);
            else store_floats_part(out + lo + j, cols - j, x);
        }
        which ^= 1;
        if constexpr (BIAS) {  // the other tile's marks, which nobody reads any more
            for (int i = tid; i < a.tile / 16; i += kLogitsThreads) s.marks[which * (a.tile / 16) + i] = 0;
            if (tid == 0) s_several[which] = 0;
        }
        if constexpr (HISTORY || BIAS) __syncthreads();
    }
}

// Workgroups per row: those that take the fewest rounds of 2 per CU times tiles, counting a tile for a workgroup's start (2 also where LDS has room for one).  256 rows of 16 tiles: 2 parts 57 us,
// 4 60, 8 63, 16 68.
static int32_t row_parts(int32_t rows, int32_t tiles) {
    const int64_t slots = 2 * kCus;
    const int32_t most = (int32_t)std::min<int64_t>(tiles, std::max<int64_t>(1, 2 * slots / rows));
    if (most > 64) return most;  // a few rows that are very long
    int32_t best = 1;
    int64_t least = INT64_MAX;
    for (int32_t p = 1; p <= most; ++p) {
        const int64_t cost = (rows * (int64_t)p + slots - 1) / slots * ((tiles + p - 1) / p + 1);
        if (cost < least) {
            least = cost;
            best = p;
        }
    }
    return best;
}

scorch_status_t launch_logits(int32_t rows, int32_t vocab, const void *in, int32_t type, int64_t ldi, const scorch_logits_rules_t &rules,
                              void *out, int32_t out_type, int64_t ldo, hipStream_t stream) {
    LogitsArgs a{in, out, rules, ldi, ldo, rows, vocab, 0, 0, 0};
    a.tile = kLogitsThreads * kLogitsVectors * (type == SCORCH_TYPE_F32 || out_type == SCORCH_TYPE_F32 ? 4 : 8);  // kPer16 of the types
    a.tiles = (int32_t)(((int64_t)vocab + a.tile - 1) / a.tile);
    a.parts = row_parts(rows, a.tiles);
    const int64_t grid = (int64_t)rows * a.parts;
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
