// Rotary positions with several axes (included by gt_attn.hip inside its
// anonymous namespace): pairs (x, y) of a head's elements are turned by
// t = pos[node][axis] theta^-e, in every head alike:
//     (x, y) <- (x cos t - y sin t, x sin t + y cos t)
// The angle is formed and reduced to a part of a turn in 64 bits.

constexpr int kRopeAxes = 4;
constexpr int kRopeMaxD = 512;

struct RopeParams {
    const float* pos;
    const void* Q;
    const void* K;
    void* outQ;
    void* outK;
    int64_t N;
    int32_t H, D;
    int32_t axes;
    int32_t dims[kRopeAxes];
    int32_t layout;
    int32_t turned;     // sum of dims
    double log2_theta;
    float sign;  // -1: turn back
};

// The pair p of a head: its elements, axis and frequency in turns.
struct RopePair {
    int32_t lo, hi, axis;
    double freq;
};

__device__ __forceinline__ RopePair rope_pair(const RopeParams& r, int p) {
    RopePair q{0, 0, 0, 0.0};
    int off = 0;
#pragma unroll
    for (int a = 0; a < kRopeAxes; ++a) {
        if (a >= r.axes) break;
        const int w = r.dims[a], k = p - off / 2;
        if (k >= 0 && k < w / 2) {
            q.axis = a;
            if (r.layout == GT_ROPE_PAIRS) {
                q.lo = off + 2 * k;
                q.hi = q.lo + 1;
            } else if (r.layout == GT_ROPE_HALVES) {
                q.lo = off + k;
                q.hi = q.lo + w / 2;
            } else {
                q.lo = p;
                q.hi = p + r.turned / 2;
            }
            const double e = r.layout == GT_ROPE_SECTIONS ? 2.0 * p / r.turned : 2.0 * k / w;
            q.freq = exp2(-e * r.log2_theta) * 0.15915494309189533577;  // 1 / (2 pi)
        }
        off += w;
    }
    return q;
}

// One thread per node and pair.
template <typename T>
__global__ void __launch_bounds__(kBlock) gt_rope_kernel(RopeParams r) {
    typedef typename Raw<T>::type R;
    const int half = r.turned / 2;
    const int64_t node = blockIdx.x;
    for (int p = threadIdx.x; p < half; p += kBlock) {
        const RopePair q = rope_pair(r, p);
        double turns = (double)r.pos[node * r.axes + q.axis] * q.freq;
        turns -= rint(turns);
        float sn, cs;
        sincospif(2.0f * (float)turns, &sn, &cs);
        sn *= r.sign;
        for (int t = 0; t < 2; ++t) {
            const R* src = static_cast<const R*>(t ? r.K : r.Q);
            R* dst = static_cast<R*>(t ? r.outK : r.outQ);
            if (!src) continue;
            for (int h = 0; h < r.H; ++h) {
                const int64_t at = (node * r.H + h) * r.D;
                const float x = to_f32(src[at + q.lo]), y = to_f32(src[at + q.hi]);
                from_f32(x * cs - y * sn, dst[at + q.lo]);
                from_f32(x * sn + y * cs, dst[at + q.hi]);
            }
        }
    }
    const int rest = r.D - r.turned;
    for (int t = 0; t < 2; ++t) {
        const R* src = static_cast<const R*>(t ? r.K : r.Q);
        R* dst = static_cast<R*>(t ? r.outK : r.outQ);
        if (!src || src == dst) continue;
        for (int i = threadIdx.x; i < rest * r.H; i += kBlock) {
            const int64_t at = (node * r.H + i / rest) * r.D + r.turned + i % rest;
            dst[at] = src[at];
        }
    }
}

gt_status run_rope(gt_dtype dtype, const float* pos, const void* Q, const void* K, void* outQ, void* outK, int64_t N,
                   int32_t H, int32_t D, const gt_rope_spec* spec, int32_t inverse, hipStream_t stream) {
    t_last_error.clear();
    if (dtype != GT_DTYPE_F32 && dtype != GT_DTYPE_BF16) return fail(GT_ERROR_NOT_SUPPORTED, "unknown dtype");
    if (N < 0 || N >= (int64_t(1) << 31)) return fail(GT_ERROR_INVALID_VALUE, "N must be in [0, 2^31)");
    if (H < 1 || D < 1) return fail(GT_ERROR_INVALID_VALUE, "H and D must be positive");
    if (D % 2 != 0 || D > kRopeMaxD || (int64_t)H * D > 65536)
        return fail(GT_ERROR_NOT_SUPPORTED, "unsupported (H, D) = (" + std::to_string(H) + ", " + std::to_string(D) +
                                                "); D even, at most " + std::to_string(kRopeMaxD) + ", H * D at most 65536");
    if (!spec) return fail(GT_ERROR_INVALID_VALUE, "spec is null");
    if (spec->axes < 1 || spec->axes > kRopeAxes) return fail(GT_ERROR_INVALID_VALUE, "spec: axes must be 1 to 4");
    if (spec->layout != GT_ROPE_PAIRS && spec->layout != GT_ROPE_HALVES && spec->layout != GT_ROPE_SECTIONS)
        return fail(GT_ERROR_NOT_SUPPORTED, "spec: unknown layout");
    if (!(std::isfinite(spec->theta) && spec->theta > 0.0)) return fail(GT_ERROR_INVALID_VALUE, "spec: theta must be positive and finite");
    RopeParams r{};
    for (int a = 0; a < spec->axes; ++a) {
        const int32_t w = spec->dims[a];
        if (w < 2 || w % 2 != 0 || w > D - r.turned)
            return fail(GT_ERROR_INVALID_VALUE, "spec: dims must be even, at least 2, and together at most D");
        r.dims[a] = w;
        r.turned += w;
    }
    if ((K == nullptr) != (outK == nullptr)) return fail(GT_ERROR_INVALID_VALUE, "K and outK must both be given, or neither");
    if (N == 0) return GT_SUCCESS;
    if (!pos || reinterpret_cast<uintptr_t>(pos) % 4 != 0) return fail(GT_ERROR_INVALID_VALUE, "pos must be non-null and 4-byte aligned");
    if (!Q || !outQ) return fail(GT_ERROR_INVALID_VALUE, "Q and outQ must be non-null");
    for (const void* ptr : {Q, K, static_cast<const void*>(outQ), static_cast<const void*>(outK)})
        if (reinterpret_cast<uintptr_t>(ptr) % 16 != 0) return fail(GT_ERROR_INVALID_VALUE, "Q, K, outQ and outK must be 16-byte aligned");
    const size_t bytes = (size_t)N * H * D * (dtype == GT_DTYPE_F32 ? 4 : 2), pb = (size_t)N * spec->axes * sizeof(float);
    if (overlaps(outQ, bytes, pos, pb) || (outK && overlaps(outK, bytes, pos, pb)))
        return fail(GT_ERROR_INVALID_VALUE, "an output overlaps pos");
    if ((outQ != Q && overlaps(outQ, bytes, Q, bytes)) || (K && overlaps(outQ, bytes, K, bytes)) ||
        (K && ((outK != K && overlaps(outK, bytes, K, bytes)) || overlaps(outK, bytes, Q, bytes) || overlaps(outK, bytes, outQ, bytes))))
        return fail(GT_ERROR_INVALID_VALUE, "an output overlaps another tensor (only its own input may be the same)");
    int dev = 0;
    if (const gt_status ds = call_device(stream, &dev); ds != GT_SUCCESS) return ds;
    r.pos = pos;
    r.Q = Q;
    r.K = K;
    r.outQ = outQ;
    r.outK = outK;
    r.N = N;
    r.H = H;
    r.D = D;
    r.axes = spec->axes;
    r.layout = (int32_t)spec->layout;
    r.log2_theta = std::log2(spec->theta);
    r.sign = inverse ? -1.0f : 1.0f;
    for (int64_t n0 = 0; n0 < N; n0 += 1 << 23) {  // (a launch holds fewer than 2^32 threads)
        RopeParams s = r;
        const int64_t at = n0 * H * D * (dtype == GT_DTYPE_F32 ? 4 : 2);
        s.pos += n0 * r.axes;
        s.Q = static_cast<const char*>(Q) + at;
        s.K = K ? static_cast<const char*>(K) + at : nullptr;
        s.outQ = static_cast<char*>(outQ) + at;
        s.outK = outK ? static_cast<char*>(outK) + at : nullptr;
        s.N = N - n0 < (1 << 23) ? N - n0 : 1 << 23;
        if (dtype == GT_DTYPE_F32)
            hipLaunchKernelGGL(gt_rope_kernel<float>, dim3((unsigned)s.N), dim3(kBlock), 0, stream, s);
        else
            hipLaunchKernelGGL(gt_rope_kernel<bf16_tag>, dim3((unsigned)s.N), dim3(kBlock), 0, stream, s);
        const hipError_t he = hipGetLastError();
        if (he != hipSuccess) return hip_fail(he, "rotary launch");
    }
    return GT_SUCCESS;
}
