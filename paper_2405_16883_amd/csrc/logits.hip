// Logits of the next token before it is chosen: penalties for tokens of the history, biases and grammar masks (definition in
// scorch_spmm.h).
//
// Bound by the bytes of the logits read and written.  A workgroup has a tile of columns of one row, for which it counts in LDS how often
// each token occurs in the row's history, and looks up the biases; then it passes over the tile once.  Counts are whole numbers, so the
// order of the atomic additions changes nothing.  Biases of one token are added by the first entry's thread, in the order of the list.
#include "device_util.h"
#include "vocab_util.h"

#include <algorithm>

namespace scorch {

constexpr int kLogitsThreads = 1024;
constexpr uint32_t kSeen = 1u << 31;    // beside the count: the token occurs anywhere in the history
constexpr uint32_t kNoBias = ~0u;
constexpr uint32_t kTwice = 1u << 31;   // beside the first bias entry of a token: there are more

struct LogitsArgs {
    const void *in;
    void *out;
    scorch_logits_rules_t rules;
    int64_t ldi, ldo;
    int32_t rows, vocab;
    int32_t tile, tiles;  // columns per workgroup, a multiple of 32
};

template <typename TI, typename TO>
__global__ __launch_bounds__(kLogitsThreads) void logits_kernel(const LogitsArgs a) {
    constexpr int N = kPer16<TI, TO>;
    extern __shared__ uint32_t s_lds[];
    const scorch_logits_rules_t &r = a.rules;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / a.tiles;
    const int32_t lo = (int32_t)(blockIdx.x % a.tiles) * a.tile;
    const int32_t cols = std::min(a.tile, a.vocab - lo);
    uint32_t *s_count = s_lds;                                      // bit 31: in the history; the others: how often from generated_from on
    uint32_t *s_bias = s_lds + (r.history_rowptr ? a.tile : 0);     // first entry of the column, as an offset into the row's list
    if (r.history_rowptr)
        for (int i = tid; i < cols; i += kLogitsThreads) s_count[i] = 0;
    if (r.bias_rowptr)
        for (int i = tid; i < cols; i += kLogitsThreads) s_bias[i] = kNoBias;
    __syncthreads();
    float repetition = 1.f, presence = 0.f, frequency = 0.f;
    if (r.history_rowptr) {
        const int32_t p0 = r.history_rowptr[row], n = r.history_rowptr[row + 1] - p0;
        const int32_t from = r.generated_from ? r.generated_from[row] : 0;
        if (r.repetition) repetition = r.repetition[row];
        if (r.presence) presence = r.presence[row];
        if (r.frequency) frequency = r.frequency[row];
        for (int32_t p = tid; p < n; p += kLogitsThreads) {
            const int32_t token = r.history[p0 + p];
            if ((uint32_t)token >= (uint32_t)a.vocab || (uint32_t)(token - lo) >= (uint32_t)cols) continue;
            if (p >= from) atomicAdd(&s_count[token - lo], 1u);
            atomicOr(&s_count[token - lo], kSeen);
        }
    }
    const int32_t b0 = r.bias_rowptr ? r.bias_rowptr[row] : 0, nb = r.bias_rowptr ? r.bias_rowptr[row + 1] - b0 : 0;
    for (int32_t p = tid; p < nb; p += kLogitsThreads) {
        const int32_t token = r.bias_tokens[b0 + p];
        if ((uint32_t)token < (uint32_t)a.vocab && (uint32_t)(token - lo) < (uint32_t)cols) atomicMin(&s_bias[token - lo], (uint32_t)p);
    }
    __syncthreads();
    for (int32_t p = tid; p < nb; p += kLogitsThreads) {
        const int32_t token = r.bias_tokens[b0 + p];
        if ((uint32_t)token < (uint32_t)a.vocab && (uint32_t)(token - lo) < (uint32_t)cols && (s_bias[token - lo] & ~kTwice) != (uint32_t)p)
            atomicOr(&s_bias[token - lo], kTwice);
    }
    __syncthreads();
    const TI *in = static_cast<const TI *>(a.in) + row * a.ldi + lo;
    TO *out = static_cast<TO *>(a.out) + row * a.ldo + lo;
    const uint32_t *mask = r.mask ? r.mask + row * r.ldm + lo / 32 : nullptr;
    for (int j = tid * N; j < cols; j += kLogitsThreads * N) {
        const int n = std::min(N, cols - j);
        float x[N];
        if (n == N) load_floats(in + j, x);
        else load_floats_part(in + j, n, 0.f, x);
        const uint32_t allowed = mask ? mask[j >> 5] >> (j & 31) : ~0u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i >= n) break;
            if (r.history_rowptr) {
                const uint32_t c = s_count[j + i];
                if (c) {
                    if (r.repetition) x[i] = x[i] > 0.f ? x[i] / repetition : x[i] * repetition;
                    const uint32_t times = c & ~kSeen;
                    if (times) x[i] = x[i] - frequency * (float)times - presence;
                }
            }
            if (r.bias_rowptr) {
                const uint32_t b = s_bias[j + i];
                if (b != kNoBias) {
                    const int32_t first = (int32_t)(b & ~kTwice);
                    float sum = r.bias_vals[b0 + first];
                    if (b & kTwice)
                        for (int32_t p = first + 1; p < nb; ++p)
                            if (r.bias_tokens[b0 + p] == lo + j + i) sum += r.bias_vals[b0 + p];
                    x[i] += sum;
                }
            }
            if (!(allowed >> i & 1)) x[i] = -INFINITY;
        }
        if (n == N) store_floats(out + j, x);
        else store_floats_part(out + j, n, x);
    }
}

scorch_status_t launch_logits(int32_t rows, int32_t vocab, const void *in, int32_t type, int64_t ldi, const scorch_logits_rules_t &rules,
                              void *out, int32_t out_type, int64_t ldo, hipStream_t stream) {
    LogitsArgs a{in, out, rules, ldi, ldo, rows, vocab, 8192, 0};
    a.tiles = (vocab + a.tile - 1) / a.tile;
    const uint32_t lds = (uint32_t)a.tile * 4 * ((rules.history_rowptr != nullptr) + (rules.bias_rowptr != nullptr));
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
                 hipLaunchKernelGGL((logits_kernel<TI, TO>), dim3((uint32_t)grid), dim3(kLogitsThreads), lds, stream, a);
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
