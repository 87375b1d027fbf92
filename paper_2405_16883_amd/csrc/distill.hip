// Distillation from a teacher's top logits: the Kullback-Leibler divergence of a row of dense logits from a short list of stored ones,
// and its gradient (definitions in scorch_spmm.h).
//
//     log sum_j exp(x z_j) = x M + log S,    M = max z_j,  S = sum_j exp(x (z_j - M)),    q_j = exp(x (z_j - M)) / S
//
// Bound by the bytes of the logits: the loss reads them once, the gradient reads and writes them.  A workgroup has a row.  Differences
// from the largest logit are formed before they are scaled: nothing overflows where the result is a number.  Loss and gradient at once keep
// the row in registers between the passes (maximum, sum, gradient), 16 or 20 vectors a thread with 16 wavefronts per CU: 81 920 16-bit columns, of
// longer rows the rest is read again.  4096 rows of 131 072 bf16: 450 us, a copy of the same bytes 417; 1.42 times the logits come in from behind L2.  Read
// again throughout 543; fewer vectors and 32 wavefronts 568; a row per CU, held whole by 1024 threads, 505.  8192 rows of 32 000: 205 us, the copy 201.
// The loss alone reads 5.7 TB/s, the gradient alone moves 5.0.
//
// The gradient is dense, c (q_j - P_j), with P_j = 0 in all but the teacher's columns.  These are marked in a bitmap in LDS: a pass over the row
// stores the others, vector by vector, and the threads that have the teacher's entries store theirs.  No element is written twice, so dZ
// may be Z.  A second bitmap marks columns that the row stores more than once; their entries are then searched for and added in order, a pass over
// the list for each (2048 rows of 32 000, 1000 entries in pairs: 765 us, 86 if distinct).
#include "device_util.h"
#include "vocab_util.h"

#include <algorithm>

namespace scorch {

constexpr float kLog2e = 1.44269504088896340736f;

enum { kDistillLoss = 1, kDistillGradient = 2 };  // what a kernel computes; both: 3

struct DistillArgs {
    const void *Z;
    void *dZ;
    const int32_t *rowptr, *colidx;
    const float *vals, *dloss;
    float *loss, *stats;
    int64_t ldz, lddz;
    int32_t rows, vocab;
    float x;       // 1 / temperature
    int32_t part;  // the gradient alone: columns per workgroup, a power of two
};

// exp(x (v - top)) for v <= top.  v - top may pass the largest number, 3.4e38, where x times it does not; it then stands for a share of 0, which is right
// while x times 3.4e38 is more than 102, as e^-102 is less than any number of 32 bits.  HALVES, for smaller x: differences of half the logits, which are
// the same otherwise.  Not for all x, because it costs the fused call of 4096 rows of 131 072 1.5 %.
constexpr float kHalvesBelow = 3e-37f;
template <bool HALVES> struct Share {
    float k;
    __device__ __forceinline__ explicit Share(float x) : k(HALVES ? 2.f * (x * kLog2e) : x * kLog2e) {}
    __device__ __forceinline__ float operator()(float v, float top) const {
        return __builtin_amdgcn_exp2f((HALVES ? fmaf(v, 0.5f, -0.5f * top) : v - top) * k);
    }
};

struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// Over all lanes whose numbers differ in bits below LANES only
template <int LANES, typename OP> __device__ __forceinline__ float lanes_all(float v, OP op) {
    if constexpr (LANES > 1) v = op(v, lane_xor<1>(v));
    if constexpr (LANES > 2) v = op(v, lane_xor<2>(v));
    if constexpr (LANES > 4) v = op(v, lane_xor<4>(v));
    if constexpr (LANES > 8) v = op(v, lane_xor<8>(v));
    if constexpr (LANES > 16) v = op(v, lane_xor<16>(v));
    if constexpr (LANES > 32) v = op(v, lane_xor<32>(v));
    return v;
}
// Over all threads of the workgroup, two values at a time; s: LDS of two values per wavefront that nothing else uses.
template <int WAVES, typename OP> __device__ __forceinline__ void block_all(float &u, float &v, OP op, float (&s)[2][WAVES]) {
    u = lanes_all<kWave>(u, op);
    v = lanes_all<kWave>(v, op);
    if constexpr (WAVES > 1) {
        const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
        if (lane == 0) {
            s[0][wv] = u;
            s[1][wv] = v;
        }
        __syncthreads();
        u = lanes_all<WAVES>(s[0][lane & (WAVES - 1)], op);
        v = lanes_all<WAVES>(s[1][lane & (WAVES - 1)], op);
    }
}

// A row of logits in vectors at multiples of 16 bytes, of which every thread keeps the first HELD in registers; what is behind them is read again
// by every pass.  The columns before the first vector and behind the last, fewer than threads, are one each of the first threads.  (Vectors from the
// row's first column on, wherever that is: 131 071 columns of 16 bits 18 % slower.)
template <typename T, int THREADS, int HELD> struct LogitRow {
    static constexpr int N = 16 / sizeof(T);
    static constexpr int kStep = THREADS * N;
    const T *z;        // at the first vector
    int32_t whole;     // columns in vectors
    int32_t skip;      // columns before them
    int32_t extra;     // this thread's column outside them, counted from the first vector
    bool has_extra;
    float extra_z;
    raw16 held[HELD > 0 ? HELD : 1];

    __device__ __forceinline__ LogitRow(const T *row, int32_t vocab) {
        skip = std::min(vocab, (int32_t)(-reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T)));
        z = row + skip;
        whole = (vocab - skip) / N * N;
        const int32_t t = (int32_t)threadIdx.x;
        has_extra = t < vocab - whole;  // neither side passes 32 bits, whatever vocab is
        extra = !has_extra ? 0 : t < skip ? t - skip : whole + (t - skip);
        extra_z = has_extra ? (float)z[extra] : -INFINITY;
#pragma unroll
        for (int u = 0; u < HELD; ++u) held[u] = holds(u) ? load_raw16(mine(z, u)) : nothing();
    }
    // Where this thread's vector u is in a row: the row's address is the same for all lanes, the offset takes one register for all u.
    template <typename P> static __device__ __forceinline__ P *mine(P *row, int u) {
        return reinterpret_cast<P *>(reinterpret_cast<uintptr_t>(row + u * kStep) + threadIdx.x * 16u);
    }
    // -infinity throughout: without a share
    static __device__ __forceinline__ raw16 nothing() {
        const uint32_t w = sizeof(T) == 4 ? 0xff800000u : std::is_same_v<T, bf16> ? 0xff80ff80u : 0xfc00fc00u;
        return raw16{w, w, w, w};
    }
    // Between passes: without it, the compiler keeps the floats of the held vectors from pass to pass, in twice the registers.
    __device__ __forceinline__ void forget_floats() {
#pragma unroll
        for (int u = 0; u < HELD; ++u) asm volatile("" : "+v"(held[u]));
    }
    __device__ __forceinline__ bool holds(int u) const { return u * kStep + (int)threadIdx.x * N < whole; }
    // f(first column counted from the first vector, where that is in `to`, vector) for all vectors of this thread
    template <typename F> __device__ __forceinline__ void each(T *to, F f) const {
        const int32_t j0 = (int)threadIdx.x * N;
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            if (holds(u)) f(u * kStep + j0, mine(to, u), held[u]);
            __builtin_amdgcn_sched_barrier(0);  // one after the other: what is not held has to fit into few registers
        }
        for (int32_t j = HELD * kStep + j0; j < whole; j += kStep) f(j, to + j, load_raw16(z + j));
    }
    // The largest logit of this thread among those that are not held, and the sum of the shares relative to it over them; not a number if there is
    // one that is not.
    template <typename SHARE> __device__ __forceinline__ void sum_with_max(SHARE share, float &top, float &sum) const {
        constexpr int U = HELD > 0 ? 8 / N : 4;  // vectors in flight
        top = extra_z == extra_z ? extra_z : -INFINITY;
        sum = extra_z == extra_z ? (extra_z == -INFINITY ? 0.f : share(extra_z, extra_z)) : NAN;
        for (int64_t j0 = HELD * kStep + (int)threadIdx.x * N; j0 < whole; j0 += U * kStep) {
            raw16 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = j0 + u * kStep < whole ? load_raw16(z + j0 + u * kStep) : nothing();
            float m = top;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i) m = fmaxf(m, element<T>(v[u], i));
            if (m == -INFINITY) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (element<T>(v[u], i) != element<T>(v[u], i)) sum = NAN;
                continue;
            }
            sum *= share(top, m);
            top = m;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i) sum += share(element<T>(v[u], i), m);
        }
    }
};

// Words for a bit per column, from bit 32 less what stands before the first vector on.
__host__ __device__ constexpr int mark_words(int32_t cols) { return (cols + 31) / 32 + 1; }

// A workgroup has a row (the gradient alone: `part` columns of one, blockIdx.y-th).
template <typename T, int WHAT, int THREADS, int HELD, bool HALVES>
__global__ __launch_bounds__(THREADS, HELD > 4 ? 4 : 8) void distill_kernel(const DistillArgs a) {
    typedef LogitRow<T, THREADS, HELD> Row;
    constexpr int N = Row::N;
    constexpr int kWaves = THREADS / kWave;
    constexpr bool kLoss = WHAT & kDistillLoss, kGradient = WHAT & kDistillGradient;
    extern __shared__ uint32_t s_marks[];  // gradient: a bit per column with an entry, then one per column with several
    __shared__ float s_red[3][2][kWaves];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const int32_t lo = kLoss ? 0 : (int32_t)blockIdx.y * a.part;
    const int32_t cols = kLoss ? a.vocab : std::min(a.part, a.vocab - lo);
    Row z(static_cast<const T *>(a.Z) + row * a.ldz + lo, cols);
    const int32_t p0 = a.rowptr[row], p1 = a.rowptr[row + 1];
    const Share<HALVES> share(a.x);
    const int words = kGradient ? mark_words(cols) : 0;
    uint32_t *s_twice = s_marks + words;
    auto bit_of = [&](int32_t col) { return (uint32_t)(col - z.skip + 32); };  // a vector's bits are in one word
    // An entry that counts as stored; col < 0 or >= cols: a column of another part.
    struct Entry {
        int32_t p, col;
        float t, z;
        bool stored;
    };
    auto read = [&](int32_t p) {
        Entry e{p, a.colidx[p], a.vals[p], 0.f, false};
        e.stored = (uint32_t)e.col < (uint32_t)a.vocab && e.t != -INFINITY;
        e.col -= lo;
        if (e.stored && (kLoss || (uint32_t)e.col < (uint32_t)cols)) e.z = (float)z.z[e.col - z.skip];
        return e;
    };
    const bool any = tid < p1 - p0;
    const Entry own = any ? read(p0 + tid) : Entry{};  // most rows have no more than one per thread: read once
    auto entries = [&](auto f) {
        if (!any) return;
        if (own.stored) f(own);
        for (int32_t p = p0 + tid; p1 - p > THREADS;) {
            p += THREADS;
            const Entry e = read(p);
            if (e.stored) f(e);
        }
    };
    if constexpr (kGradient) {
        for (int i = tid; i < 2 * words; i += THREADS) s_marks[i] = 0;
        __syncthreads();
    }
    float t_top = -INFINITY;
    entries([&](const Entry &e) {
        t_top = fmaxf(t_top, e.t);
        if constexpr (kGradient) {
            if ((uint32_t)e.col >= (uint32_t)cols) return;
            const uint32_t b = bit_of(e.col), bit = 1u << (b & 31);
            if (atomicOr(&s_marks[b >> 5], bit) & bit) atomicOr(&s_twice[b >> 5], bit);
        }
    });
    // largest logits, of the student's row and of the stored entries, then the sums
    float top = -INFINITY, sum = 0.f, z_top = 0.f;
    if constexpr (kLoss) {
        z.sum_with_max(share, top, sum);
        z_top = top;
#pragma unroll
        for (int u = 0; u < HELD; ++u)
            if (z.holds(u))
#pragma unroll
                for (int i = 0; i < N; ++i) z_top = fmaxf(z_top, element<T>(z.held[u], i));
    }
    z.forget_floats();
    block_all(z_top, t_top, Max(), s_red[0]);
    if constexpr (kLoss) {
        sum = top == -INFINITY ? sum : sum * share(top, z_top);
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            if (z.holds(u))
#pragma unroll
                for (int i = 0; i < N; ++i) sum += share(element<T>(z.held[u], i), z_top);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    z.forget_floats();
    float t_sum = 0.f;
    entries([&](const Entry &e) { t_sum += share(e.t, t_top); });
    block_all(sum, t_sum, Sum(), s_red[1]);
    const bool none = t_sum == 0.f;  // otherwise the largest entry's share is 1, or something is not a number
    if constexpr (!kLoss) {
        z_top = a.stats[2 * row];
        sum = a.stats[2 * row + 1];
    }
    const float t_scale = 1.f / t_sum;
    if constexpr (kLoss) {
        const float log_sums = logf(t_sum) - logf(sum);
        float divergence = 0.f, unused = 0.f;
        entries([&](const Entry &e) {
            const float prob = share(e.t, t_top) * t_scale;
            // prob x ((t - t_top) - (z - z_top)) - prob log_sums, in an order in which only the product itself can pass the largest number or vanish
            const float apart = fmaf(e.t, 0.5f, -0.5f * t_top) - fmaf(e.z, 0.5f, -0.5f * z_top);
            if (prob != 0.f) divergence += 2.f * (apart * fminf(a.x, 1.f) * (prob * fmaxf(a.x, 1.f))) - prob * log_sums;
        });
        block_all(divergence, unused, Sum(), s_red[2]);
        if (tid == 0) {
            a.loss[row] = divergence;
            if (!kGradient) {
                a.stats[2 * row] = z_top;
                a.stats[2 * row + 1] = sum;
            }
        }
    }
    if constexpr (kGradient) {
        T *dz = static_cast<T *>(a.dZ) + row * a.lddz + lo;
        const float c = (a.dloss ? a.dloss[row] : 1.f) * a.x;
        const float q_scale = 1.f / sum, cq = c * q_scale;
        entries([&](const Entry &e) {
            if ((uint32_t)e.col >= (uint32_t)cols) return;
            float prob = share(e.t, t_top) * t_scale;
            if (s_twice[bit_of(e.col) >> 5] >> (bit_of(e.col) & 31) & 1) {
                // the column's first entry adds them all up, in their order, and is the only one to write there; the list is the same for all lanes
                bool first = true;
                prob = 0.f;
#pragma unroll 4
                for (int32_t o = p0; o < p1; ++o) {
                    const float t = a.vals[o];
                    const bool same = (a.colidx[o] - lo == e.col) & (t != -INFINITY);
                    first &= !same | (o >= e.p);
                    prob += same ? share(t, t_top) * t_scale : 0.f;
                }
                if (!first) return;
            }
            dz[e.col] = (T)(c * (share(e.z, z_top) * q_scale - prob));
        });
        // Streaming stores: written once, and the memory-side cache is left to the logits that are read again
        z.each(dz + z.skip, [&](int32_t j, T *to, const raw16 &v) {
            const uint32_t marks = s_marks[(j >> 5) + 1] >> (j & 31) & ((1u << N) - 1);
            float y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = none ? 0.f : cq * share(element<T>(v, i), z_top);
            if (marks == 0) {
                store_floats<T, N, true>(to, y);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (!(marks >> i & 1)) to[i] = (T)y[i];
            }
        });
        const uint32_t b = (uint32_t)(z.extra + 32);
        if (z.has_extra && !(s_marks[b >> 5] >> (b & 31) & 1))
            dz[z.skip + z.extra] = (T)(none ? 0.f : cq * share(z.extra_z, z_top));
    }
}

template <typename T, int WHAT, int THREADS, int HELD, bool HALVES = false> static void launch_distill_as(const DistillArgs &a, hipStream_t stream) {
    const int32_t part = WHAT == kDistillGradient ? a.part : std::max(a.vocab, 1);
    const uint32_t lds = WHAT & kDistillGradient ? (uint32_t)mark_words(part) * 8 : 0;
    hipLaunchKernelGGL((distill_kernel<T, WHAT, THREADS, HELD, HALVES>), dim3((uint32_t)a.rows, WHAT == kDistillGradient ? (uint32_t)((a.vocab + part - 1) / part) : 1), dim3(THREADS), lds,
                       stream, a);
}

// Threads per row: as many as fill the chip.  1 row of 131 072: 1024 threads 10 us, 256 threads 15; 2048 rows of 32 000: 256 threads 24 us.  Short rows of
// many: a wavefront each (8192 rows of 1000: 7 us, 256 threads 17).
template <typename T> static void launch_distill_loss(const DistillArgs &a, hipStream_t stream) {
    if (a.x < kHalvesBelow) launch_distill_as<T, kDistillLoss, 1024, 0, true>(a, stream);
    else if (a.rows >= 8 * kCus && a.vocab <= 4096) launch_distill_as<T, kDistillLoss, 64, 0>(a, stream);
    else if (a.rows >= 8 * kCus) launch_distill_as<T, kDistillLoss, 256, 0>(a, stream);
    else if (a.rows >= 4 * kCus) launch_distill_as<T, kDistillLoss, 512, 0>(a, stream);
    else launch_distill_as<T, kDistillLoss, 1024, 0>(a, stream);
}

// Columns per workgroup: rows are cut until there are 8 workgroups per CU (1 row of 131 072: 4 us, whole 34), and so that the marks leave room for that
// many in LDS (2048 rows of 262 144: 422 us, whole 574).
template <typename T> static void launch_distill_gradient(DistillArgs a, hipStream_t stream) {
    a.part = 65536;
    while (a.part / 2 >= a.vocab) a.part /= 2;
    while (a.part > 4096 && (int64_t)a.rows * ((a.vocab + a.part - 1) / a.part) < 8 * kCus) a.part /= 2;
    if (a.x < kHalvesBelow) launch_distill_as<T, kDistillGradient, 256, 0, true>(a, stream);
    else if (a.rows >= 8 * kCus && a.vocab <= 4096) launch_distill_as<T, kDistillGradient, 64, 0>(a, stream);
    else launch_distill_as<T, kDistillGradient, 256, 0>(a, stream);
}

// The fewest threads whose registers hold the row, so that many rows are at work on a CU; with no more rows than CUs as many threads as a row takes
// (256 rows of 131 072: 32 us, 512 threads 38).  Rows are never cut here: 1 to 64 rows of 131 072 take 20 us, loss and gradient in two calls 13 to 17.
// 512 threads with 20 vectors spill 5 registers and were the fastest of the forms tried for long rows all the same.
template <typename T> static void launch_distill_both(const DistillArgs &a, hipStream_t stream) {
    constexpr int kBoth = kDistillLoss | kDistillGradient;
    constexpr int64_t kPer = 16 / sizeof(T);
    if (a.x < kHalvesBelow) {
        launch_distill_as<T, kBoth, 1024, 0, true>(a, stream);
    } else if (a.rows <= kCus) {  // a row per CU: as many threads as it takes
        if (a.vocab <= 1024 * 4 * kPer) launch_distill_as<T, kBoth, 1024, 4>(a, stream);
        else launch_distill_as<T, kBoth, 1024, 16>(a, stream);
    } else if (a.vocab <= 64 * 4 * kPer) launch_distill_as<T, kBoth, 64, 4>(a, stream);
    else if (a.vocab <= 256 * 4 * kPer) launch_distill_as<T, kBoth, 256, 4>(a, stream);
    else if (a.vocab <= 256 * 16 * kPer) launch_distill_as<T, kBoth, 256, 16>(a, stream);
    else if (a.vocab <= 512 * 16 * kPer) launch_distill_as<T, kBoth, 512, 16>(a, stream);
    else launch_distill_as<T, kBoth, 512, 20>(a, stream);
}

scorch_status_t launch_distill(int what, int32_t rows, int32_t vocab, const void *Z, int32_t z_type, int64_t ldz, const int32_t *rowptr,
                               const int32_t *colidx, const float *vals, float x, const float *dloss, float *loss, float *stats,
                               void *dZ, int64_t lddz, hipStream_t stream) {
    const DistillArgs a{Z, dZ, rowptr, colidx, vals, dloss, loss, stats, ldz, lddz, rows, vocab, x, 0};
    if (!grid_fits(rows, 1024)) {
        set_error("distillation: %d rows need a larger launch than HIP takes", rows);
        return SCORCH_ERR_UNSUPPORTED;
    }
    const bool ok = with_type(z_type, [&](auto tz) {
        typedef typename decltype(tz)::type T;
        if (what == kDistillLoss) launch_distill_loss<T>(a, stream);
        else if (what == kDistillGradient) launch_distill_gradient<T>(a, stream);
        else launch_distill_both<T>(a, stream);
    });
    if (!ok) {
        set_error("distillation: unknown type %d", z_type);
        return SCORCH_ERR_INVALID_ARG;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "launch distill_kernel");
    return SCORCH_OK;
}

}  // namespace scorch
