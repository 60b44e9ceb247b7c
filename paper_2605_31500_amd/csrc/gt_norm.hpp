// Layer norm over rows of F elements, forward and backward (included by
// gt_attn.hip inside its anonymous namespace):
//     mean = sum x / F, rstd = 1 / sqrt(sum (x - mean)^2 / F + eps)
//     out  = (x - mean) rstd gamma + beta
//     dX   = rstd (g - mean(g) - x^ mean(g x^)),  g = dout gamma, x^ = (x - mean) rstd
//     dgamma = sum over rows of dout x^, dbeta = sum over rows of dout

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

// One wavefront per row.
template <typename T>
__global__ void __launch_bounds__(kBlock) gt_norm_fwd_kernel(NormArgs a) {
    typedef typename Raw<T>::type R;
    const int lane = threadIdx.x & (kWave - 1);
    for (int64_t row = (int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / kWave; row < a.N; row += (int64_t)gridDim.x * kWavesPerBlock) {
    const R* x = static_cast<const R*>(a.X) + row * a.F;
    R* y = static_cast<R*>(a.out) + row * a.F;
    float s = 0.0f;
    for (int f = lane; f < a.F; f += kWave) s += to_f32(x[f]);
    const float mean = head_sum<64>(s) / (float)a.F;
    float v = 0.0f;
    for (int f = lane; f < a.F; f += kWave) {
        const float d = to_f32(x[f]) - mean;
        v = fmaf(d, d, v);
    }
    const float rstd = 1.0f / sqrtf(head_sum<64>(v) / (float)a.F + a.eps);
    for (int f = lane; f < a.F; f += kWave) {
        const float h = (to_f32(x[f]) - mean) * rstd;
        from_f32(fmaf(h, a.gamma ? a.gamma[f] : 1.0f, a.beta ? a.beta[f] : 0.0f), y[f]);
    }
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    }
}

template <typename T>
__global__ void __launch_bounds__(kBlock) gt_norm_bwd_kernel(NormArgs a) {
    typedef typename Raw<T>::type R;
    const int lane = threadIdx.x & (kWave - 1);
    for (int64_t row = (int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / kWave; row < a.N; row += (int64_t)gridDim.x * kWavesPerBlock) {
    const R* x = static_cast<const R*>(a.X) + row * a.F;
    const R* dy = static_cast<const R*>(a.dout) + row * a.F;
    R* dx = static_cast<R*>(a.out) + row * a.F;
    const float mean = a.mean_in[row], rstd = a.rstd_in[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int f = lane; f < a.F; f += kWave) {
        const float g = to_f32(dy[f]) * (a.gamma ? a.gamma[f] : 1.0f);
        s1 += g;
        s2 = fmaf(g, (to_f32(x[f]) - mean) * rstd, s2);
    }
    s1 = head_sum<64>(s1) / (float)a.F;
    s2 = head_sum<64>(s2) / (float)a.F;
    for (int f = lane; f < a.F; f += kWave) {
        const float g = to_f32(dy[f]) * (a.gamma ? a.gamma[f] : 1.0f), h = (to_f32(x[f]) - mean) * rstd;
        from_f32(rstd * (g - s1 - h * s2), dx[f]);
    }
    }
}

// Parameters' gradients: a workgroup sums a stretch of rows for 64 columns,
// the second kernel the stretches.
constexpr int kNormStretches = 256;

template <typename T>
__global__ void __launch_bounds__(kBlock) gt_norm_param_kernel(NormArgs a, float* part) {
    typedef typename Raw<T>::type R;
    __shared__ float sums[2][kWavesPerBlock][kWave];
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int f = blockIdx.x * kWave + lane;
    const int64_t lo = a.N * blockIdx.y / gridDim.y, hi = a.N * (blockIdx.y + 1) / gridDim.y;
    float sg = 0.0f, sb = 0.0f;
    if (f < a.F)
        for (int64_t i = lo + wv; i < hi; i += kWavesPerBlock) {
            const float dy = to_f32(static_cast<const R*>(a.dout)[i * a.F + f]);
            const float x = to_f32(static_cast<const R*>(a.X)[i * a.F + f]);
            sg = fmaf(dy, (x - a.mean_in[i]) * a.rstd_in[i], sg);
            sb += dy;
        }
    sums[0][wv][lane] = sg;
    sums[1][wv][lane] = sb;
    __syncthreads();
    if (wv < 2 && f < a.F)
        part[((int64_t)blockIdx.y * 2 + wv) * a.F + f] =
            (sums[wv][0][lane] + sums[wv][1][lane]) + (sums[wv][2][lane] + sums[wv][3][lane]);
}

__global__ void __launch_bounds__(kBlock) gt_norm_param_sum_kernel(const float* part, int stretches, int32_t F, float* dgamma,
                                                                   float* dbeta) {
    const int f = blockIdx.x * kBlock + threadIdx.x;
    if (f >= F) return;
    double sg = 0.0, sb = 0.0;
    for (int s = 0; s < stretches; ++s) {
        sg += part[(int64_t)s * 2 * F + f];
        sb += part[((int64_t)s * 2 + 1) * F + f];
    }
    if (dgamma) dgamma[f] = (float)sg;
    if (dbeta) dbeta[f] = (float)sb;
}

template <typename T>
gt_status launch_norm_fwd(const NormArgs& a, hipStream_t stream) {
    const int64_t blocks = std::min<int64_t>((a.N + kWavesPerBlock - 1) / kWavesPerBlock, 1 << 20);
    hipLaunchKernelGGL(gt_norm_fwd_kernel<T>, dim3((unsigned)blocks), dim3(kBlock), 0, stream, a);
    const hipError_t he = hipGetLastError();
    return he == hipSuccess ? GT_SUCCESS : hip_fail(he, "layer norm launch");
}

template <typename T>
gt_status launch_norm_bwd(const NormArgs& a, int dev, hipStream_t stream) {
    hipError_t he = hipSuccess;
    if (a.dgamma || a.dbeta) {
        // (before dX, which may be one of its inputs)
        const int stretches = (int)(a.N < kNormStretches ? a.N : kNormStretches);
        CallWorkspace cw;
        if (const gt_status st = acquire_workspace(dev, (size_t)(stretches > 0 ? stretches : 1) * 2 * a.F * sizeof(float), stream, cw);
            st != GT_SUCCESS)
            return st;
        float* part = reinterpret_cast<float*>(cw.ptr);
        if (stretches > 0) {
            hipLaunchKernelGGL(gt_norm_param_kernel<T>, dim3((a.F + kWave - 1) / kWave, stretches), dim3(kBlock), 0, stream, a, part);
            if ((he = hipGetLastError()) != hipSuccess) return hip_fail(he, "layer norm parameter launch");
        }
        hipLaunchKernelGGL(gt_norm_param_sum_kernel, dim3((a.F + kBlock - 1) / kBlock), dim3(kBlock), 0, stream, part, stretches, a.F,
                           a.dgamma, a.dbeta);
        if ((he = hipGetLastError()) != hipSuccess) return hip_fail(he, "layer norm parameter launch");
    }
    if (a.N == 0) return GT_SUCCESS;
    const int64_t blocks = std::min<int64_t>((a.N + kWavesPerBlock - 1) / kWavesPerBlock, 1 << 20);
    hipLaunchKernelGGL(gt_norm_bwd_kernel<T>, dim3((unsigned)blocks), dim3(kBlock), 0, stream, a);
    he = hipGetLastError();
    return he == hipSuccess ? GT_SUCCESS : hip_fail(he, "layer norm backward launch");
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
    if (!backward) return dtype == GT_DTYPE_F32 ? launch_norm_fwd<float>(a, stream) : launch_norm_fwd<bf16_tag>(a, stream);
    return dtype == GT_DTYPE_F32 ? launch_norm_bwd<float>(a, dev, stream) : launch_norm_bwd<bf16_tag>(a, dev, stream);
}
