// Layer norm over rows of F elements, forward and backward (included by
// gt_attn.hip inside its anonymous namespace):
//     mean = sum x / F, rstd = 1 / sqrt(sum (x - mean)^2 / F + eps)
//     out  = (x - mean) rstd gamma + beta
//     dX   = rstd (g - mean(g) - x^ mean(g x^)),  g = dout gamma, x^ = (x - mean) rstd
//     dgamma = sum over rows of dout x^, dbeta = sum over rows of dout
// A row is read once and kept in registers between its sums and its output, so a
// call moves what it has to and is bound by HBM (1 M rows of 256 bf16 elements:
// forward 198 us, 5.5 TB/s; 169 K rows of 512 fp32: backward 183 us, 5.7 TB/s, of
// which the parameters' gradients' second kernel is 3), small calls by their
// launches (2000 rows of 128 fp32: 3.9 us).

struct NormArgs {
    const void* X;
    const void* dout;
    const float* gamma;
    const float* beta;
    const float* mean_in;
    const float* rstd_in;
    void* out;  // out, or dX
    float* mean;
    float* rstd;
    float* dgamma;
    float* dbeta;
    int64_t N;
    int32_t F;
    float eps;
};

constexpr int32_t kNormMaxF = 16384;

// A row is read once, into registers, by G lanes with K accesses of W elements
// each: 16 bytes where rows are a whole number of them (NORM_WHOLE), else 4 bytes
// (NORM_WORDS).  Rows of an odd number of bf16 elements (NORM_PHASE) are read in
// 16-byte accesses all the same: a row starts inside one, `phase` elements of the
// row before it are read along and masked, and its first and last access store
// single elements; a group's rows are all of one phase, so that its accesses hold
// the same columns in every row.  (fp32 and even bf16 rows by phases / by words,
// us, forward and backward: 309 K rows of 818 bf16 441 / 210, 522 / 311; 11 K of 3121
// fp32 58 / 49, 157 / 90.  100 K rows of 819 bf16 by phases: forward 145 with a
// wavefront for a row and 107 with four, backward 177 and 221.)
enum { NORM_WHOLE, NORM_WORDS, NORM_PHASE };

template <int BYTES> struct NormAccess;
template <> struct NormAccess<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct NormAccess<4> { typedef uint32_t type; };

template <typename T, int G_, int K_, int MODE>
struct NormRow {
    static_assert(MODE != NORM_PHASE || std::is_same<T, bf16_tag>::value, "fp32 rows are whole words");
    static constexpr bool kPhase = MODE == NORM_PHASE;
    static constexpr int kBytes = MODE == NORM_WORDS ? 4 : 16;
    static constexpr int G = G_, K = K_, W = kBytes / Elt<T>::kBytes, kDwords = kBytes / 4;
    static constexpr int kThreads = G > kBlock ? G : kBlock;
    static constexpr int kGroups = kThreads / G;  // of a workgroup
    // rows that a group requests together
    static constexpr int kAhead = G > kWave ? 1 : MODE == NORM_WORDS ? (K <= 4 ? 4 : 2) : K > 2 ? 1 : 4 / K;
    static constexpr int kAheadBwd = K * W > 8 ? 1 : kPhase ? (kAhead + 1) / 2 : kAhead;
    // parameters stay in registers (read again for every row, us: backward of 60 K rows of
    // 1000 bf16 113 against 77)
    static constexpr bool kKeep = K * W <= (kPhase ? 16 : 32);
    typedef typename NormAccess<kBytes>::type Vec;
    Vec v[K];

    // Column of the first element of access k.
    __device__ __forceinline__ static int column(int lig, int k, int phase) { return (lig + k * G) * W - (kPhase ? phase : 0); }
    __device__ __forceinline__ static bool holds(int col, int e, int32_t F) {
        return kPhase ? (uint32_t)(col + e) < (uint32_t)F : col < F;
    }
    __device__ __forceinline__ static uint32_t dword(const Vec& x, int d) {
        if constexpr (kDwords == 1)
            return x;
        else
            return x[d];
    }

    // (elements of other rows are read as 0)
    __device__ __forceinline__ void load(const void* base, int64_t N, int64_t row, int32_t F, int lig, int phase) {
        typedef typename Raw<T>::type R;
        const R* p = static_cast<const R*>(base) + row * F;
        const int64_t left = (N - row) * F;  // elements up to the tensor's end
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = column(lig, k, phase);
            v[k] = Vec{};
            if (c >= F || (kPhase && c + W <= 0)) continue;
            const Vec* at = reinterpret_cast<const Vec*>(p + c);
            if constexpr (kPhase) {
                uint32_t mask[kDwords];
#pragma unroll
                for (int d = 0; d < kDwords; ++d)
                    mask[d] = (holds(c, 2 * d, F) ? 0x0000FFFFu : 0u) | (holds(c, 2 * d + 1, F) ? 0xFFFF0000u : 0u);
                if (c + W > left) {  // (nothing past the end)
#pragma unroll
                    for (int e = 0; e < W; ++e)
                        if (holds(c, e, F)) v[k][e / 2] |= (uint32_t)p[c + e] << (e % 2 * 16);
                } else {
                    v[k] = *at;
#pragma unroll
                    for (int d = 0; d < kDwords; ++d) v[k][d] &= mask[d];
                }
            } else {
                // past the caches, unless two rows share lines (plain loads throughout / past
                // the caches, us: backward of 169 K rows of 512 fp32 194 / 183, of 60 K rows of
                // 203 bf16 26.0 / 31.0; a choice at run time costs the former 9)
                v[k] = MODE == NORM_WHOLE ? __builtin_nontemporal_load(at) : *at;
            }
        }
    }

    __device__ __forceinline__ void elements(int k, float (&x)[W]) const {
#pragma unroll
        for (int e = 0; e < W; ++e)
            if constexpr (std::is_same<T, float>::value)
                x[e] = __uint_as_float(dword(v[k], e));
            else
                x[e] = __uint_as_float(e % 2 ? dword(v[k], e / 2) & 0xFFFF0000u : dword(v[k], e / 2) << 16);
    }

    __device__ __forceinline__ static void store(void* base, int64_t row, int32_t F, int lig, int phase, int k, const float (&x)[W]) {
        typedef typename Raw<T>::type R;
        R* p = static_cast<R*>(base) + row * F;
        const int c = column(lig, k, phase);
        if (c >= F || (kPhase && c + W <= 0)) return;
        uint32_t o[kDwords];
#pragma unroll
        for (int d = 0; d < kDwords; ++d)
            if constexpr (std::is_same<T, float>::value)
                o[d] = __float_as_uint(x[d]);
            else
                o[d] = pack_bf16(x[2 * d], x[2 * d + 1]);
        Vec y;
        __builtin_memcpy(&y, o, sizeof y);
        Vec* at = reinterpret_cast<Vec*>(p + c);
        if constexpr (MODE == NORM_WHOLE) {
            __builtin_nontemporal_store(y, at);
        } else {  // (rows share lines: left to the L2 to put together)
            if (!kPhase || (c >= 0 && c + W <= F))
                *at = y;
            else
#pragma unroll
                for (int e = 0; e < W; ++e)
                    if (holds(c, e, F)) p[c + e] = (R)(o[e / 2] >> (e % 2 * 16));
        }
    }

    // Parameters at access k (`other` where there are none).
    __device__ __forceinline__ static void params(const float* base, int32_t F, int lig, int phase, int k, float other, float (&x)[W]) {
        const int c = column(lig, k, phase);
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = base && holds(c, e, F) ? base[c + e] : other;
    }
};

// The rows of a group: `first` and every `step` after it, and with each of them
// the next ones `apart`.  A workgroup's rows follow one another, unless those of
// a group would be of different phases then (the grid is a multiple of 8).
// (Rows that a group requests together apart by the grid, fp32 and bf16 alike:
// 1 M rows of 256 bf16 elements 214 us against 198.)
template <typename Row, int AHEAD>
struct NormRows {
    static constexpr bool kTogether = !Row::kPhase || Row::kGroups % Row::W == 0;
    int64_t first, step, apart;
    int phase;
    __device__ __forceinline__ NormRows(int32_t F, int g) {
        first = (int64_t)blockIdx.x * Row::kGroups * (kTogether ? AHEAD : 1) + g;
        step = (int64_t)gridDim.x * Row::kGroups * AHEAD;
        apart = kTogether ? Row::kGroups : (int64_t)gridDim.x * Row::kGroups;
        phase = Row::kPhase ? (int)((first % Row::W) * (F % Row::W) % Row::W) : 0;
    }
};

// Sums of M values over the G lanes of a row's group, in every lane.
template <int G, int M>
__device__ __forceinline__ void group_sum(float (&x)[M], float* lds, int& turn) {
    if constexpr (G <= kWave) {
#pragma unroll
        for (int m = 0; m < M; ++m) x[m] = head_sum<G>(x[m]);
    } else {
        // (two buffers in turn: a sum's readers are done before the next but one is written)
        constexpr int kWaves = G / kWave;
        float* buf = lds + turn * kWaves * M;
        turn ^= 1;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            x[m] = head_sum<kWave>(x[m]);
            if (threadIdx.x % kWave == 0) buf[m * kWaves + threadIdx.x / kWave] = x[m];
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < M; ++m) {
            x[m] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) x[m] += buf[m * kWaves + w];
        }
    }
}

template <typename T, int G, int K, int MODE>
__global__ void __launch_bounds__((NormRow<T, G, K, MODE>::kThreads)) gt_norm_fwd_kernel(NormArgs a) {
    using Row = NormRow<T, G, K, MODE>;
    constexpr int W = Row::W;
    constexpr int kAhead = Row::kAhead;
    __shared__ float lds[G > kWave ? 2 * G / kWave : 1];
    int turn = 0;
    const int lig = threadIdx.x % G, g = threadIdx.x / G;
    const float inv_f = 1.0f / (float)a.F;
    const NormRows<Row, kAhead> rows(a.F, g);
    constexpr bool kKeep = Row::kKeep;
    float gm[kKeep ? K : 1][W], bt[kKeep ? K : 1][W];
    if constexpr (kKeep)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            Row::params(a.gamma, a.F, lig, rows.phase, k, 1.0f, gm[k]);
            Row::params(a.beta, a.F, lig, rows.phase, k, 0.0f, bt[k]);
        }
    // (uniform where the group is more than a wavefront)
    for (int64_t r0 = rows.first; r0 < a.N; r0 += rows.step) {
        Row x[kAhead];
#pragma unroll
        for (int b = 0; b < kAhead; ++b) {
            const int64_t row = r0 + b * rows.apart;
            x[b].load(a.X, a.N, row < a.N ? row : r0, a.F, lig, rows.phase);
        }
#pragma unroll
        for (int b = 0; b < kAhead; ++b) {
            const int64_t row = r0 + b * rows.apart;
            float s[1] = {0.0f};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float e[W];
                x[b].elements(k, e);
#pragma unroll
                for (int i = 0; i < W; ++i) s[0] += e[i];
            }
            group_sum<G, 1>(s, lds, turn);
            const float mean = s[0] * inv_f;
            float q[1] = {0.0f};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float e[W];
                x[b].elements(k, e);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float d = Row::holds(Row::column(lig, k, rows.phase), i, a.F) ? e[i] - mean : 0.0f;
                    q[0] = fmaf(d, d, q[0]);
                }
            }
            group_sum<G, 1>(q, lds, turn);
            const float rstd = 1.0f / sqrtf(fmaf(q[0], inv_f, a.eps));
            if (row >= a.N) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float e[W], o[W];
                x[b].elements(k, e);
                if constexpr (!kKeep) {
                    Row::params(a.gamma, a.F, lig, rows.phase, k, 1.0f, gm[0]);
                    Row::params(a.beta, a.F, lig, rows.phase, k, 0.0f, bt[0]);
                }
#pragma unroll
                for (int i = 0; i < W; ++i) o[i] = fmaf((e[i] - mean) * rstd, gm[kKeep ? k : 0][i], bt[kKeep ? k : 0][i]);
                Row::store(a.out, row, a.F, lig, rows.phase, k, o);
            }
            if (lig == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        }
    }
}

// Backward.  A group sums its rows' shares of the parameters' gradients in
// registers; at the end they are added over the groups of the workgroup, which
// leaves one partial row each of dgamma and dbeta in `part` [workgroup][2][F].
template <typename T, int G, int K, int MODE>
__global__ void __launch_bounds__((NormRow<T, G, K, MODE>::kThreads)) gt_norm_bwd_kernel(NormArgs a, float* part) {
    using Row = NormRow<T, G, K, MODE>;
    constexpr int W = Row::W;
    constexpr int kAhead = Row::kAheadBwd;
    constexpr int kLdsSum = G > kWave ? 4 * G / kWave : 0, kLdsParam = Row::kGroups > 1 ? Row::kThreads * K * W : 0;
    __shared__ float lds[kLdsSum > kLdsParam ? kLdsSum : kLdsParam > 0 ? kLdsParam : 1];
    int turn = 0;
    const int lig = threadIdx.x % G, g = threadIdx.x / G;
    const float inv_f = 1.0f / (float)a.F;
    float sg[K][W], sb[K][W];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < W; ++i) sg[k][i] = sb[k][i] = 0.0f;
    const NormRows<Row, kAhead> rows(a.F, g);
    constexpr bool kKeep = Row::kKeep;
    float gm[kKeep ? K : 1][W];
    if constexpr (kKeep)
#pragma unroll
        for (int k = 0; k < K; ++k) Row::params(a.gamma, a.F, lig, rows.phase, k, 1.0f, gm[k]);
    // (uniform where the group is more than a wavefront)
    for (int64_t r0 = rows.first; r0 < a.N; r0 += rows.step) {
        Row x[kAhead], y[kAhead];
        float mean[kAhead], rstd[kAhead];
#pragma unroll
        for (int b = 0; b < kAhead; ++b) {
            const int64_t row = r0 + b * rows.apart, at = row < a.N ? row : r0;
            x[b].load(a.X, a.N, at, a.F, lig, rows.phase);
            y[b].load(a.dout, a.N, at, a.F, lig, rows.phase);
            mean[b] = a.mean_in[at];
            rstd[b] = a.rstd_in[at];
        }
#pragma unroll
        for (int b = 0; b < kAhead; ++b) {
            const int64_t row = r0 + b * rows.apart;
            if (row >= a.N) break;
            // x^ = x rstd - mean rstd (as near as the rounded mean itself is)
            const float shift = -mean[b] * rstd[b];
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float ex[W], ey[W];
                x[b].elements(k, ex);
                y[b].elements(k, ey);
                if constexpr (!kKeep) Row::params(a.gamma, a.F, lig, rows.phase, k, 1.0f, gm[0]);
#pragma unroll
                for (int i = 0; i < W; ++i) {  // (dout is 0 outside the row)
                    const float h = fmaf(ex[i], rstd[b], shift), gr = ey[i] * gm[kKeep ? k : 0][i];
                    s[0] += gr;
                    s[1] = fmaf(gr, h, s[1]);
                    sg[k][i] = fmaf(ey[i], h, sg[k][i]);
                    sb[k][i] += ey[i];
                }
            }
            group_sum<G, 2>(s, lds, turn);
            const float m1 = -rstd[b] * (s[0] * inv_f), m2 = -rstd[b] * (s[1] * inv_f);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float ex[W], ey[W], o[W];
                x[b].elements(k, ex);
                y[b].elements(k, ey);
                if constexpr (!kKeep) Row::params(a.gamma, a.F, lig, rows.phase, k, 1.0f, gm[0]);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float h = fmaf(ex[i], rstd[b], shift), gr = ey[i] * gm[kKeep ? k : 0][i];
                    o[i] = fmaf(gr, rstd[b], fmaf(h, m2, m1));
                }
                Row::store(a.out, row, a.F, lig, rows.phase, k, o);
            }
        }
    }
    if (!part) return;
    float* dst = part + (int64_t)blockIdx.x * 2 * a.F;
    if constexpr (Row::kGroups == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = Row::column(lig, k, rows.phase);
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (Row::holds(c, i, a.F)) {
                    dst[c + i] = sg[k][i];
                    dst[a.F + c + i] = sb[k][i];
                }
        }
    } else {
        constexpr int kCols = G * K * W;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = Row::column(lig, k, rows.phase);
#pragma unroll
                for (int i = 0; i < W; ++i)
                    if (Row::holds(c, i, a.F)) lds[g * kCols + c + i] = which ? sb[k][i] : sg[k][i];
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.F; c += Row::kThreads) {
                float x = lds[c];
                for (int o = 1; o < Row::kGroups; ++o) x += lds[o * kCols + c];
                dst[which * a.F + c] = x;
            }
        }
    }
}

// The workgroups' partial rows, added in 64 bits in a fixed order: 16 columns
// (a 64-byte piece of every row) and 64 stretches of the rows to a workgroup.
constexpr int kNormCols = 16, kNormStretches = 64;

__global__ void __launch_bounds__(kNormCols * kNormStretches)
gt_norm_param_kernel(const float* part, int blocks, int32_t F, float* dgamma, float* dbeta) {
    __shared__ double sums[kNormStretches][kNormCols];
    const int c = threadIdx.x % kNormCols, r = threadIdx.x / kNormCols, col = blockIdx.x * kNormCols + c;
    double s = 0.0;
    if (col < 2 * F)
#pragma unroll 8
        for (int b = r; b < blocks; b += kNormStretches) s += part[(int64_t)b * 2 * F + col];
    sums[r][c] = s;
    __syncthreads();
    if (r < kNormCols) {
#pragma unroll
        for (int i = kNormCols; i < kNormStretches; i += kNormCols) s += sums[r + i][c];
        sums[r][c] = s;
    }
    __syncthreads();
    if (r != 0 || col >= 2 * F) return;
#pragma unroll
    for (int i = 1; i < kNormCols; ++i) s += sums[i][c];
    float* dst = col < F ? dgamma : dbeta;
    if (dst) dst[col < F ? col : col - F] = (float)s;
}

// Workgroups: all that the device holds at once (each keeps its parameters and
// sums for many rows), or one for the rows that its groups request together.
template <typename T, int G, int K, int MODE, bool BACKWARD>
int norm_blocks(int64_t rows_per_block, int64_t N, int dev) {
    static std::atomic<int> cache[64];
    int most = dev >= 0 && dev < 64 ? cache[dev].load() : 0;
    if (most == 0) {
        int nb = 0;
        const void* kernel = BACKWARD ? reinterpret_cast<const void*>(gt_norm_bwd_kernel<T, G, K, MODE>)
                                      : reinterpret_cast<const void*>(gt_norm_fwd_kernel<T, G, K, MODE>);
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&nb, kernel, NormRow<T, G, K, MODE>::kThreads, 0) != hipSuccess || nb <= 0) nb = 1;
        most = nb * device_cus(dev);
        if (dev >= 0 && dev < 64) cache[dev] = most;
    }
    int64_t need = (N + rows_per_block - 1) / rows_per_block;
    if (need > most) need = most;
    return (int)(MODE == NORM_PHASE ? (need + 7) / 8 * 8 : need);
}

template <typename T, int G, int K, int MODE>
gt_status launch_norm_fwd(const NormArgs& a, int dev, hipStream_t stream) {
    using Row = NormRow<T, G, K, MODE>;
    const int blocks = norm_blocks<T, G, K, MODE, false>(Row::kGroups * Row::kAhead, a.N, dev);
    hipLaunchKernelGGL((gt_norm_fwd_kernel<T, G, K, MODE>), dim3(blocks), dim3(Row::kThreads), 0, stream, a);
    const hipError_t he = hipGetLastError();
    return he == hipSuccess ? GT_SUCCESS : hip_fail(he, "layer norm launch");
}

template <typename T, int G, int K, int MODE>
gt_status launch_norm_bwd(const NormArgs& a, int dev, hipStream_t stream) {
    using Row = NormRow<T, G, K, MODE>;
    hipError_t he = hipSuccess;
    const int blocks = norm_blocks<T, G, K, MODE, true>(Row::kGroups * Row::kAheadBwd, a.N, dev);
    CallWorkspace cw;
    if (a.dgamma || a.dbeta)
        if (const gt_status st = acquire_workspace(dev, (size_t)blocks * 2 * a.F * sizeof(float), stream, cw); st != GT_SUCCESS) return st;
    float* part = reinterpret_cast<float*>(cw.ptr);
    hipLaunchKernelGGL((gt_norm_bwd_kernel<T, G, K, MODE>), dim3(blocks), dim3(Row::kThreads), 0, stream, a, part);
    if ((he = hipGetLastError()) != hipSuccess) return hip_fail(he, "layer norm backward launch");
    if (part) {
        hipLaunchKernelGGL(gt_norm_param_kernel, dim3((2 * a.F + kNormCols - 1) / kNormCols), dim3(kNormCols * kNormStretches), 0, stream, part, blocks, a.F,
                           a.dgamma, a.dbeta);
        if ((he = hipGetLastError()) != hipSuccess) return hip_fail(he, "layer norm parameter launch");
    }
    return GT_SUCCESS;
}

template <typename T, int G, int K, int MODE>
gt_status launch_norm(const NormArgs& a, bool backward, int dev, hipStream_t stream) {
    return backward ? launch_norm_bwd<T, G, K, MODE>(a, dev, stream) : launch_norm_fwd<T, G, K, MODE>(a, dev, stream);
}

// The lanes of a row by its accesses.  A wavefront takes rows of a few accesses
// per lane, since a row of more wavefronts waits for their sums; the masks of
// phases cost registers, which get more lanes instead.
template <typename T>
gt_status pick_whole(const NormArgs& a, bool backward, int dev, hipStream_t stream) {
    constexpr int M = NORM_WHOLE;
    const int32_t c = a.F / NormRow<T, 8, 1, M>::W;
    if (c <= 4) return launch_norm<T, 4, 1, M>(a, backward, dev, stream);
    if (c <= 8) return launch_norm<T, 8, 1, M>(a, backward, dev, stream);
    if (c <= 16) return launch_norm<T, 16, 1, M>(a, backward, dev, stream);
    if (c <= 32) return launch_norm<T, 32, 1, M>(a, backward, dev, stream);
    if (c <= 64) return launch_norm<T, 64, 1, M>(a, backward, dev, stream);
    if (c <= 128) return launch_norm<T, 64, 2, M>(a, backward, dev, stream);
    if (c <= 256) return launch_norm<T, 64, 4, M>(a, backward, dev, stream);
    if (c <= 512) return launch_norm<T, 256, 2, M>(a, backward, dev, stream);
    if (c <= 1024) return launch_norm<T, 256, 4, M>(a, backward, dev, stream);
    if constexpr (std::is_same<T, float>::value)
        if (c > 2048) return launch_norm<T, 1024, 4, M>(a, backward, dev, stream);
    return launch_norm<T, 512, 4, M>(a, backward, dev, stream);
}

template <typename T>
gt_status pick_words(const NormArgs& a, bool backward, int dev, hipStream_t stream) {
    constexpr int M = NORM_WORDS;
    const int32_t c = a.F / NormRow<T, 8, 1, M>::W;
    if (c <= 8) return launch_norm<T, 8, 1, M>(a, backward, dev, stream);
    if (c <= 16) return launch_norm<T, 16, 1, M>(a, backward, dev, stream);
    if (c <= 32) return launch_norm<T, 32, 1, M>(a, backward, dev, stream);
    if (c <= 64) return launch_norm<T, 64, 1, M>(a, backward, dev, stream);
    if (c <= 128) return launch_norm<T, 64, 2, M>(a, backward, dev, stream);
    if (c <= 256) return launch_norm<T, 64, 4, M>(a, backward, dev, stream);
    if (c <= 512) return launch_norm<T, 64, 8, M>(a, backward, dev, stream);
    if (c <= 1024) return launch_norm<T, 256, 4, M>(a, backward, dev, stream);
    if (c <= 2048) return launch_norm<T, 256, 8, M>(a, backward, dev, stream);
    if (c <= 4096) return launch_norm<T, 512, 8, M>(a, backward, dev, stream);
    if constexpr (std::is_same<T, float>::value)
        if (c > 8192) return launch_norm<T, 1024, 16, M>(a, backward, dev, stream);
    return launch_norm<T, 1024, 8, M>(a, backward, dev, stream);
}

gt_status pick_phase(const NormArgs& a, bool backward, int dev, hipStream_t stream) {
    typedef bf16_tag T;
    constexpr int M = NORM_PHASE;
    const int32_t c = (a.F + 14) / 8;  // (with the largest phase)
    if (c <= 4) return launch_norm<T, 4, 1, M>(a, backward, dev, stream);
    if (c <= 8) return launch_norm<T, 8, 1, M>(a, backward, dev, stream);
    if (c <= 16) return launch_norm<T, 16, 1, M>(a, backward, dev, stream);
    if (c <= 32) return launch_norm<T, 32, 1, M>(a, backward, dev, stream);
    if (c <= 64) return launch_norm<T, 64, 1, M>(a, backward, dev, stream);
    if (c <= 128 && backward) return launch_norm_bwd<T, 64, 2, M>(a, dev, stream);
    if (c <= 256) return launch_norm<T, 256, 1, M>(a, backward, dev, stream);
    if (c <= 512) return launch_norm<T, 512, 1, M>(a, backward, dev, stream);
    if (c <= 1024) return launch_norm<T, 1024, 1, M>(a, backward, dev, stream);
    return launch_norm<T, 1024, 3, M>(a, backward, dev, stream);
}

template <typename T>
gt_status dispatch_norm(const NormArgs& a, bool backward, int dev, hipStream_t stream) {
    if (a.N == 0) {  // (0.0f is all bits 0)
        for (float* p : {a.dgamma, a.dbeta})
            if (p)
                if (const hipError_t he = clear_counters(reinterpret_cast<int32_t*>(p), a.F, stream); he != hipSuccess)
                    return hip_fail(he, "layer norm parameter launch");
        return GT_SUCCESS;
    }
    const int64_t bytes = (int64_t)a.F * Elt<T>::kBytes;
    if (bytes % 16 == 0) return pick_whole<T>(a, backward, dev, stream);
    if constexpr (std::is_same<T, bf16_tag>::value)
        if (bytes % 4 != 0) return pick_phase(a, backward, dev, stream);
    return pick_words<T>(a, backward, dev, stream);
}

gt_status run_norm(gt_dtype dtype, const NormArgs& a, bool backward, hipStream_t stream) {
    t_last_error.clear();
    if (dtype != GT_DTYPE_F32 && dtype != GT_DTYPE_BF16) return fail(GT_ERROR_NOT_SUPPORTED, "unknown dtype");
    if (a.N < 0 || a.N >= (int64_t(1) << 31)) return fail(GT_ERROR_INVALID_VALUE, "N must be in [0, 2^31)");
    if (a.F < 1) return fail(GT_ERROR_INVALID_VALUE, "F must be positive");
    if (a.F > kNormMaxF) return fail(GT_ERROR_NOT_SUPPORTED, "unsupported F = " + std::to_string(a.F) + "; at most " + std::to_string(kNormMaxF));
    if (!backward && !(std::isfinite(a.eps) && a.eps >= 0.0f)) return fail(GT_ERROR_INVALID_VALUE, "eps must be finite and not negative");
    const size_t bytes = (size_t)a.N * a.F * (dtype == GT_DTYPE_F32 ? 4 : 2), cols = (size_t)a.F * sizeof(float),
                 rows = (size_t)a.N * sizeof(float);
    struct Buffer {
        const void* ptr;
        size_t bytes;
        const char* name;
    };
    const Buffer feats[] = {{a.X, bytes, "X"}, {a.dout, bytes, "dout"}, {a.out, bytes, backward ? "dX" : "out"}};
    const Buffer params[] = {{a.gamma, cols, "gamma"}, {a.beta, cols, "beta"}, {a.mean_in, rows, "mean"}, {a.rstd_in, rows, "rstd"}};
    const Buffer outs[] = {{a.mean, rows, "mean"}, {a.rstd, rows, "rstd"}, {a.dgamma, cols, "dgamma"}, {a.dbeta, cols, "dbeta"}};
    if (a.N > 0)
        for (const Buffer& b : feats) {
            if (&b == &feats[1] && !backward) continue;
            if (!b.ptr || reinterpret_cast<uintptr_t>(b.ptr) % 16 != 0)
                return fail(GT_ERROR_INVALID_VALUE, std::string(b.name) + " must be non-null and 16-byte aligned");
        }
    if (backward && a.N > 0 && (!a.mean_in || !a.rstd_in)) return fail(GT_ERROR_INVALID_VALUE, "mean and rstd must be non-null");
    for (const Buffer& b : params)
        if (reinterpret_cast<uintptr_t>(b.ptr) % 4 != 0) return fail(GT_ERROR_INVALID_VALUE, std::string(b.name) + " must be 4-byte aligned");
    for (const Buffer& b : outs)
        if (reinterpret_cast<uintptr_t>(b.ptr) % 4 != 0) return fail(GT_ERROR_INVALID_VALUE, std::string(b.name) + " must be 4-byte aligned");
    // each output against what it must not overlap (the row output may be an input itself)
    auto clash = [](const Buffer& x, const Buffer& y) { return x.ptr && y.ptr && x.bytes && y.bytes && overlaps(x.ptr, x.bytes, y.ptr, y.bytes); };
    auto refuse = [](const Buffer& x, const Buffer& y) {
        return fail(GT_ERROR_INVALID_VALUE, std::string(x.name) + " overlaps " + y.name);
    };
    const Buffer& out = feats[2];
    for (int k = 0; k < 2; ++k)
        if (out.ptr != feats[k].ptr && clash(out, feats[k])) return refuse(out, feats[k]);
    for (const Buffer& p : params)
        if (clash(out, p)) return refuse(out, p);
    for (int k = 0; k < 4; ++k) {
        for (const Buffer& f : feats)
            if (clash(outs[k], f)) return refuse(outs[k], f);
        for (const Buffer& p : params)
            if (clash(outs[k], p)) return refuse(outs[k], p);
        for (int l = 0; l < k; ++l)
            if (clash(outs[k], outs[l])) return refuse(outs[k], outs[l]);
    }
    if (a.N == 0 && !a.dgamma && !a.dbeta) return GT_SUCCESS;
    int dev = 0;
    if (const gt_status ds = call_device(stream, &dev); ds != GT_SUCCESS) return ds;
    return dtype == GT_DTYPE_F32 ? dispatch_norm<float>(a, backward, dev, stream) : dispatch_norm<bf16_tag>(a, backward, dev, stream);
}
