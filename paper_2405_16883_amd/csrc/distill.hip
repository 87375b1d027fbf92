// Distillation from a teacher's top logits: the Kullback-Leibler divergence of a row of dense logits from a short list of stored ones,
// and its gradient (definitions in scorch_spmm.h).
//
//     log sum_j exp(x z_j) = x M + log S,    M = max z_j,  S = sum_j exp(x (z_j - M)),    q_j = exp(x (z_j - M)) / S
//
// Bound by the bytes of the logits: the loss reads them once, the gradient reads and writes them.  A workgroup has a row.  Differences
// from the largest logit are formed before they are scaled, so that nothing overflows where the result is a number.
//
// The gradient is dense, c (q_j - P_j), with P_j = 0 in all but the teacher's columns.  These are marked in a bitmap in LDS: a pass over the row
// stores the others, vector by vector, and the threads that have the teacher's entries store theirs.  No element is written twice, so dZ
// may be Z.  A second bitmap marks columns that the row stores more than once; their entries are then searched for and added in order.
#include "device_util.h"
#include "vocab_util.h"

#include <algorithm>

namespace scorch {

constexpr int kDistillThreads = 1024;
constexpr int kDistillWaves = kDistillThreads / kWave;
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
    float x;  // 1 / temperature
};

struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

template <typename OP> __device__ __forceinline__ float wave_all(float v, OP op) {
    v = op(v, lane_xor<1>(v));
    v = op(v, lane_xor<2>(v));
    v = op(v, lane_xor<4>(v));
    v = op(v, lane_xor<8>(v));
    v = op(v, lane_xor<16>(v));
    return op(v, lane_xor<32>(v));
}
// Over all threads of the workgroup, two values at a time; s: LDS of two values per wavefront, free before and after.
template <typename OP> __device__ __forceinline__ void block_all(float &u, float &v, OP op, float (&s)[2][kDistillWaves]) {
    u = wave_all(u, op);
    v = wave_all(v, op);
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane == 0) {
        s[0][wv] = u;
        s[1][wv] = v;
    }
    __syncthreads();
    u = s[0][0];
    v = s[1][0];
    for (int w = 1; w < kDistillWaves; ++w) {
        u = op(u, s[0][w]);
        v = op(v, s[1][w]);
    }
    __syncthreads();
}

template <typename T, int WHAT>
__global__ __launch_bounds__(kDistillThreads) void distill_kernel(const DistillArgs a) {
    constexpr int N = 16 / sizeof(T);
    constexpr bool kLoss = WHAT & kDistillLoss, kGradient = WHAT & kDistillGradient;
    extern __shared__ uint32_t s_marks[];  // gradient: a bit per column with an entry, then one per column with several
    __shared__ float s_red[2][kDistillWaves];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.Z) + row * a.ldz;
    const int32_t p0 = a.rowptr[row], p1 = a.rowptr[row + 1];
    const float k = a.x * kLog2e;
    const int words = (a.vocab + 31) / 32;
    uint32_t *s_twice = s_marks + words;
    auto stored = [&](int32_t p, int32_t &col, float &t) {
        col = a.colidx[p];
        t = a.vals[p];
        return (uint32_t)col < (uint32_t)a.vocab && t != -INFINITY;
    };

    if constexpr (kGradient) {
        for (int i = tid; i < 2 * words; i += kDistillThreads) s_marks[i] = 0;
        __syncthreads();
    }
    // largest logits, of the student's row and of the stored entries; the sums go along with a maximum of each thread's own
    float top = -INFINITY, sum = 0.f, t_top = -INFINITY, t_any = 0.f;
    if constexpr (kLoss) {
        for (int j = tid * N; j < a.vocab; j += kDistillThreads * N) {
            float y[N];
            if (a.vocab - j >= N) load_floats(z + j, y);
            else load_floats_part(z + j, a.vocab - j, -INFINITY, y);
            float m = top;
#pragma unroll
            for (int i = 0; i < N; ++i) m = fmaxf(m, y[i]);
            if (m == -INFINITY) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (y[i] != y[i]) sum = NAN;
                continue;
            }
            sum *= __builtin_amdgcn_exp2f((top - m) * k);
            top = m;
#pragma unroll
            for (int i = 0; i < N; ++i) sum += __builtin_amdgcn_exp2f((y[i] - m) * k);
        }
    }
    for (int32_t p = p0 + tid; p < p1; p += kDistillThreads) {
        int32_t col;
        float t;
        if (!stored(p, col, t)) continue;
        t_top = fmaxf(t_top, t);
        t_any = 1.f;
        if constexpr (kGradient) {
            const uint32_t bit = 1u << (col & 31);
            if (atomicOr(&s_marks[col >> 5], bit) & bit) atomicOr(&s_twice[col >> 5], bit);
        }
    }
    float z_top = top;
    block_all(z_top, t_top, Max(), s_red);
    if constexpr (kLoss) sum = top == -INFINITY ? sum : sum * __builtin_amdgcn_exp2f((top - z_top) * k);
    float t_sum = 0.f;
    for (int32_t p = p0 + tid; p < p1; p += kDistillThreads) {
        int32_t col;
        float t;
        if (stored(p, col, t)) t_sum += __builtin_amdgcn_exp2f((t - t_top) * k);
    }
    block_all(sum, t_sum, Sum(), s_red);
    float divergence = 0.f;
    block_all(t_any, divergence, Max(), s_red);
    if constexpr (!kLoss) {
        z_top = a.stats[2 * row];
        sum = a.stats[2 * row + 1];
    }
    const float t_scale = 1.f / t_sum;
    if constexpr (kLoss) {
        const float log_sums = logf(t_sum) - logf(sum);
        for (int32_t p = p0 + tid; p < p1; p += kDistillThreads) {
            int32_t col;
            float t;
            if (!stored(p, col, t)) continue;
            const float prob = __builtin_amdgcn_exp2f((t - t_top) * k) * t_scale;
            const float zk = (float)z[col];
            if (prob != 0.f) divergence += prob * (a.x * (t - t_top) - a.x * (zk - z_top) - log_sums);
        }
        float unused = 0.f;
        block_all(divergence, unused, Sum(), s_red);
        if (tid == 0) {
            a.loss[row] = divergence;
            if (a.stats) {
                a.stats[2 * row] = z_top;
                a.stats[2 * row + 1] = sum;
            }
        }
    }
    if constexpr (kGradient) {
        T *dz = static_cast<T *>(a.dZ) + row * a.lddz;
        const float c = (a.dloss ? a.dloss[row] : 1.f) * a.x;
        const bool none = t_any == 0.f;
        const float q_scale = 1.f / sum;
        for (int32_t p = p0 + tid; p < p1; p += kDistillThreads) {
            int32_t col;
            float t;
            if (!stored(p, col, t)) continue;
            float prob = __builtin_amdgcn_exp2f((t - t_top) * k) * t_scale;
            if (s_twice[col >> 5] >> (col & 31) & 1) {
                // the column's first entry adds the others up and is the only one to read and write there
                bool first = true;
                for (int32_t o = p0; o < p && first; ++o) {
                    int32_t other;
                    first = !(stored(o, other, t) && other == col);
                }
                if (!first) continue;
                for (int32_t o = p + 1; o < p1; ++o) {
                    int32_t other;
                    if (stored(o, other, t) && other == col) prob += __builtin_amdgcn_exp2f((t - t_top) * k) * t_scale;
                }
            }
            dz[col] = (T)(c * (__builtin_amdgcn_exp2f(((float)z[col] - z_top) * k) * q_scale - prob));
        }
        for (int j = tid * N; j < a.vocab; j += kDistillThreads * N) {
            const int n = std::min(N, a.vocab - j);
            const uint32_t marks = s_marks[j >> 5] >> (j & 31) & ((1u << N) - 1);
            float y[N];
            if (n == N) load_floats(z + j, y);
            else load_floats_part(z + j, n, 0.f, y);
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = none ? 0.f : c * (__builtin_amdgcn_exp2f((y[i] - z_top) * k) * q_scale);
            if (n == N && marks == 0) {
                store_floats(dz + j, y);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i < n && !(marks >> i & 1)) dz[j + i] = (T)y[i];
            }
        }
    }
}

template <typename T, int WHAT> static void launch_distill_as(const DistillArgs &a, hipStream_t stream) {
    const uint32_t lds = WHAT & kDistillGradient ? (uint32_t)((a.vocab + 31) / 32) * 8 : 0;
    hipLaunchKernelGGL((distill_kernel<T, WHAT>), dim3((uint32_t)a.rows), dim3(kDistillThreads), lds, stream, a);
}

scorch_status_t launch_distill(int what, int32_t rows, int32_t vocab, const void *Z, int32_t z_type, int64_t ldz, const int32_t *rowptr,
                               const int32_t *colidx, const float *vals, float x, const float *dloss, float *loss, float *stats,
                               void *dZ, int64_t lddz, hipStream_t stream) {
    const DistillArgs a{Z, dZ, rowptr, colidx, vals, dloss, loss, stats, ldz, lddz, rows, vocab, x};
    if (!grid_fits(rows, kDistillThreads)) {
        set_error("distillation: %d rows need a larger launch than HIP takes", rows);
        return SCORCH_ERR_UNSUPPORTED;
    }
    const bool ok = with_type(z_type, [&](auto tz) {
        typedef typename decltype(tz)::type T;
        if (what == kDistillLoss) launch_distill_as<T, kDistillLoss>(a, stream);
        else if (what == kDistillGradient) launch_distill_as<T, kDistillGradient>(a, stream);
        else launch_distill_as<T, kDistillLoss | kDistillGradient>(a, stream);
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
