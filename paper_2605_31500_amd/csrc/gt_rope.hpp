// Rotary positions with several axes (included by gt_attn.hip inside its
// anonymous namespace): pairs (x, y) of a head's elements are turned by
// t = pos[node][axis] theta^-e, in every head alike:
//     (x, y) <- (x cos t - y sin t, x sin t + y cos t)
// The angle is formed and reduced to a part of a turn in 64 bits.  Each element is
// read and written once: bound by HBM (1 M nodes, Q and K of 8x64 bf16 by three
// axes in halves of 8 and 12 elements: 815 us, 5.3 TB/s; in whole 16-byte accesses
// the same), small calls by the chain of position, table and rows (16 K nodes of
// 4x32 fp32: 8.0 us).  Non-temporal accesses: 1089 us, since an access' lines are
// shared by the halves' other one.

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
    int32_t nodes;   // of a workgroup at a time
    int32_t copies;  // the elements past the turned ones are copied
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

// A workgroup takes `nodes` nodes at a time.  It forms their angles' sines and
// cosines once, into LDS, and then runs over their rows of Q and K with 16-byte
// accesses (W elements; 8, 4 or 2 bytes where pairs do not come in whole ones), so
// that every head's pairs share one evaluation and the rows move as in a copy.
//
// The elements of a head are turned by units: W neighbours (PAIRS), or W and
// the W elements that they are paired with.  Elements past the turned ones are
// units of their own, which are copied unless the call is in place.  What a
// unit is, the workgroup writes into LDS once.
typedef uint32_t RopeVec4 __attribute__((ext_vector_type(4)));
typedef uint32_t RopeVec2 __attribute__((ext_vector_type(2)));
template <int BYTES> struct RopeAccess;
template <> struct RopeAccess<16> { typedef RopeVec4 type; };
template <> struct RopeAccess<8> { typedef RopeVec2 type; };
template <> struct RopeAccess<4> { typedef uint32_t type; };
template <> struct RopeAccess<2> { typedef uint16_t type; };

template <typename T, int W> struct RopeUnit {
    typedef typename RopeAccess<W * Elt<T>::kBytes>::type Vec;
    __device__ __forceinline__ static void widen_to(const Vec& v, float (&x)[W]) {
        typename Raw<T>::type r[W];
        __builtin_memcpy(r, &v, sizeof v);
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = to_f32(r[e]);
    }
    __device__ __forceinline__ static Vec narrow_from(const float (&x)[W]) {
        Vec v;
        if constexpr (std::is_same<T, float>::value || W == 1) {
            typename Raw<T>::type r[W];
#pragma unroll
            for (int e = 0; e < W; ++e) from_f32(x[e], r[e]);
            __builtin_memcpy(&v, r, sizeof v);
        } else {
            uint32_t r[W / 2];
#pragma unroll
            for (int e = 0; e < W; e += 2) r[e / 2] = pack_bf16(x[e], x[e + 1]);
            __builtin_memcpy(&v, r, sizeof v);
        }
        return v;
    }
};

// Sine and cosine of `turns` whole turns: less the nearest quarter turn in 64
// bits, so that what is rounded to fp32 is at most an eighth of a turn, and then
// the Taylor polynomials in the rest's radians r, |r| <= pi / 4 (their next terms
// are below 2^-28: r^11 / 11! and r^12 / 12!).
__device__ __forceinline__ float2 rope_cos_sin(double turns) {
    const double quarters = 4.0 * turns, q = rint(quarters);
    const float r = (float)((quarters - q) * 1.5707963267948966), r2 = r * r;
    const int k = (int)(q - 4.0 * floor(0.25 * q)) & 3;  // (NaN: any)
    float s = fmaf(r2, 2.7557319e-6f, -1.9841270e-4f);
    s = fmaf(r2, s, 8.3333333e-3f);
    s = fmaf(r2, s, -1.6666667e-1f);
    s = fmaf(r * r2, s, r);
    float c = fmaf(r2, -2.7557319e-7f, 2.4801587e-5f);
    c = fmaf(r2, c, -1.3888889e-3f);
    c = fmaf(r2, c, 4.1666667e-2f);
    c = fmaf(r2, c, -0.5f);
    c = fmaf(r2, c, 1.0f);
    const float cs = k & 1 ? s : c, sn = k & 1 ? c : s;
    return make_float2(k == 1 || k == 2 ? -cs : cs, k >= 2 ? -sn : sn);
}

constexpr int kRopeTable = 2048;    // pairs' sines and cosines at a time
constexpr int kRopeHeld = 1 << 16;  // units of a tensor at a time
constexpr int kRopeUnits = 8;       // that a thread requests together

// i / d by a multiplication, for i < 2^16 and d <= 2^16 (i e < 2^32, with e <= d
// what the factor's rounding adds).
struct Quotient {
    uint32_t factor;
    __device__ __forceinline__ explicit Quotient(int d) : factor(d == 1 ? 0u : 0xFFFFFFFFu / (uint32_t)d + 1u) {}
    __device__ __forceinline__ int operator()(int i) const { return factor ? (int)__umulhi((uint32_t)i, factor) : i; }
};

template <typename T, int W, bool PAIRS>
__global__ void __launch_bounds__(kBlock) gt_rope_kernel(RopeParams r) {
    typedef typename Raw<T>::type R;
    using Unit = RopeUnit<T, W>;
    typedef typename Unit::Vec Vec;
    __shared__ float2 table[kRopeTable];
    __shared__ double freq[kRopeMaxD / 2];
    __shared__ int32_t axis[kRopeMaxD / 2];
    __shared__ int32_t first[kRopeMaxD / W], second[kRopeMaxD / W], pair[kRopeMaxD / W];  // of each unit; pair -1: copied
    const int half = r.turned / 2;
    for (int p = threadIdx.x; p < half; p += kBlock) {
        const RopePair q = rope_pair(r, p);
        freq[p] = q.freq;
        axis[p] = q.axis;
        if (PAIRS ? q.lo % W == 0 : p % W == 0) {
            const int u = PAIRS ? q.lo / W : p / W;
            first[u] = q.lo;
            second[u] = q.hi;
            pair[u] = p;
        }
    }
    const int turned_units = PAIRS ? r.turned / W : half / W, units = r.copies ? turned_units + (r.D - r.turned) / W : turned_units;
    for (int u = turned_units + threadIdx.x; u < units; u += kBlock) {
        first[u] = second[u] = r.turned + (u - turned_units) * W;
        pair[u] = -1;
    }
    const int tensors = r.K ? 2 : 1, per_node = r.H * units;
    const Quotient by_half(half), by_units(units), by_heads(r.H);
    for (int64_t n0 = (int64_t)blockIdx.x * r.nodes; n0 < r.N; n0 += (int64_t)gridDim.x * r.nodes) {
        const int nodes = (int)(r.N - n0 < r.nodes ? r.N - n0 : r.nodes);
        __syncthreads();  // (the units and frequencies are there, the table's readers done)
        for (int i = threadIdx.x; i < nodes * half; i += kBlock) {
            const int n = by_half(i), p = i - n * half;
            float2 cs = rope_cos_sin((double)r.pos[(n0 + n) * r.axes + axis[p]] * freq[p]);
            cs.y *= r.sign;
            table[i] = cs;
        }
        __syncthreads();
        // (the units of Q, then those of K: requested together)
        const int each = nodes * per_node, total = tensors * each;
        const int64_t row0 = n0 * r.H * r.D;
        for (int i0 = threadIdx.x; i0 < total; i0 += kRopeUnits * kBlock) {
            Vec a[kRopeUnits], b[PAIRS ? 1 : kRopeUnits];
            int at[kRopeUnits], bt[kRopeUnits], cs[kRopeUnits];
#pragma unroll
            for (int j = 0; j < kRopeUnits; ++j) {
                int i = i0 + j * kBlock < total ? i0 + j * kBlock : i0;  // (past the last: read and left)
                const bool key = i >= each;
                if (key) i -= each;
                const R* src = static_cast<const R*>(key ? r.K : r.Q) + row0;
                const int head = by_units(i), u = i - head * units;
                at[j] = head * r.D + first[u];
                bt[j] = head * r.D + second[u];
                cs[j] = pair[u] < 0 ? -1 : by_heads(head) * half + pair[u];
                a[j] = *reinterpret_cast<const Vec*>(src + at[j]);
                if constexpr (!PAIRS) b[j] = *reinterpret_cast<const Vec*>(src + bt[j]);
            }
#pragma unroll
            for (int j = 0; j < kRopeUnits; ++j) {
                if (i0 + j * kBlock >= total) break;
                R* dst = static_cast<R*>(i0 + j * kBlock >= each ? r.outK : r.outQ) + row0;
                if (cs[j] < 0) {
                    *reinterpret_cast<Vec*>(dst + at[j]) = a[j];
                    continue;
                }
                const float2* c = table + cs[j];
                float x[W], ox[W];
                Unit::widen_to(a[j], x);
                if constexpr (PAIRS) {
#pragma unroll
                    for (int e = 0; e < W; e += 2) {
                        ox[e] = x[e] * c[e / 2].x - x[e + 1] * c[e / 2].y;
                        ox[e + 1] = x[e] * c[e / 2].y + x[e + 1] * c[e / 2].x;
                    }
                } else {
                    float y[W], oy[W];
                    Unit::widen_to(b[j], y);
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        ox[e] = x[e] * c[e].x - y[e] * c[e].y;
                        oy[e] = x[e] * c[e].y + y[e] * c[e].x;
                    }
                    *reinterpret_cast<Vec*>(dst + bt[j]) = Unit::narrow_from(oy);
                }
                *reinterpret_cast<Vec*>(dst + at[j]) = Unit::narrow_from(ox);
            }
        }
    }
}

// Where the pairs do not come in whole accesses but heads are whole 16-byte
// vectors: a thread keeps one place in a head (W elements) for all rows of a
// node and head that it takes, and so its elements' partners and frequencies.
// Rows pass through LDS, from which it reads the partners; they still move by 16
// bytes (us, by units / so: single bf16 elements, 194 K nodes of 4x128 253 / 180,
// 241 K of 2x32 54 / 35; two bf16, 524 K of 8x64 532 / 430, but 523 K of 2x32 70 /
// 80; four bf16, 524 K of 8x64 411 / 430; two fp32, 390 K of 4x128 690 / 630).
template <typename T>
__global__ void __launch_bounds__(kBlock) gt_rope_rows_kernel(RopeParams r) {
    typedef typename Raw<T>::type R;
    constexpr int W = 16 / Elt<T>::kBytes, kRows = 2;
    using Unit = RopeUnit<T, W>;
    typedef typename Unit::Vec Vec;
    __shared__ float2 table[kRopeTable];
    __shared__ double freq[kRopeMaxD / 2];
    __shared__ int32_t axis[kRopeMaxD / 2];
    __shared__ uint32_t element[kRopeMaxD];  // partner | pair << 10 | turned << 30 | second of its pair << 31
    __shared__ __attribute__((aligned(16))) R stage[2][kRows * kBlock * W];
    const int half = r.turned / 2, vecs = r.D / W;
    for (int x = threadIdx.x; x < r.D; x += kBlock) element[x] = (uint32_t)x;
    __syncthreads();
    for (int p = threadIdx.x; p < half; p += kBlock) {
        const RopePair q = rope_pair(r, p);
        freq[p] = q.freq;
        axis[p] = q.axis;
        element[q.lo] = (uint32_t)q.hi | (uint32_t)p << 10 | 1u << 30;
        element[q.hi] = (uint32_t)q.lo | (uint32_t)p << 10 | 3u << 30;
    }
    __syncthreads();
    const int at_once = kBlock / vecs, place = threadIdx.x % vecs, mine = threadIdx.x / vecs;  // (vecs <= 128)
    const bool idle = mine >= at_once;
    uint32_t el[W];
#pragma unroll
    for (int e = 0; e < W; ++e) el[e] = element[place * W + e];
    const Quotient by_half(half), by_heads(r.H);
    for (int64_t n0 = (int64_t)blockIdx.x * r.nodes; n0 < r.N; n0 += (int64_t)gridDim.x * r.nodes) {
        const int nodes = (int)(r.N - n0 < r.nodes ? r.N - n0 : r.nodes);
        __syncthreads();
        for (int i = threadIdx.x; i < nodes * half; i += kBlock) {
            const int n = by_half(i), p = i - n * half;
            float2 cs = rope_cos_sin((double)r.pos[(n0 + n) * r.axes + axis[p]] * freq[p]);
            cs.y *= r.sign;
            table[i] = cs;
        }
        const int each = nodes * r.H, total = (r.K ? 2 : 1) * each;
        const int64_t row0 = n0 * r.H;
        for (int i0 = 0, turn = 0; i0 < total; i0 += kRows * at_once, turn ^= 1) {
            Vec v[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const int i = i0 + j * at_once + mine, k = i >= each ? i - each : i;
                if (idle || i >= total) continue;
                v[j] = *reinterpret_cast<const Vec*>(static_cast<const R*>(i >= each ? r.K : r.Q) + (row0 + k) * r.D + place * W);
                *reinterpret_cast<Vec*>(&stage[turn][(j * at_once + mine) * r.D + place * W]) = v[j];
            }
            __syncthreads();  // (rows and table are there; the other stage's readers are past the sync before)
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const int i = i0 + j * at_once + mine, k = i >= each ? i - each : i;
                if (idle || i >= total) continue;
                const R* row = &stage[turn][(j * at_once + mine) * r.D];
                const float2* cs = table + by_heads(k) * half;
                float x[W], o[W];
                Unit::widen_to(v[j], x);
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const float y = to_f32(row[el[e] & 1023u]);
                    const float2 c = cs[(el[e] >> 10) & 1023u];
                    const float turned = el[e] >> 31 ? y * c.y + x[e] * c.x : x[e] * c.x - y * c.y;
                    o[e] = el[e] >> 30 & 1u ? turned : x[e];
                }
                *reinterpret_cast<Vec*>(static_cast<R*>(i >= each ? r.outK : r.outQ) + (row0 + k) * r.D + place * W) = Unit::narrow_from(o);
            }
        }
    }
}

// Elements of an access: the most, up to 16 bytes, that divide every stretch of
// elements which lie together with their partners, and the rest of the head.
int rope_access(const RopeParams& r, int elt_bytes) {
    int w = 16 / elt_bytes;
    auto fit = [&w](int n) {
        while (n % w != 0) w /= 2;
    };
    fit(r.D);
    fit(r.D - r.turned);
    int off = 0;
    for (int a = 0; a < r.axes; ++a) {
        if (r.layout == GT_ROPE_PAIRS) {
            fit(off);
        } else if (r.layout == GT_ROPE_HALVES) {
            fit(off);
            fit(r.dims[a] / 2);
        }
        off += r.dims[a];
    }
    if (r.layout == GT_ROPE_SECTIONS) fit(off / 2);
    return w;
}

template <typename T, int W, bool PAIRS>
gt_status launch_rope(RopeParams r, int dev, hipStream_t stream) {
    // nodes of a workgroup: as many as the table holds, fewer where the call has not enough for the device
    const int64_t most = kRopeTable / (r.turned / 2), even = (r.N + 4 * device_cus(dev) - 1) / (4 * device_cus(dev));
    const int64_t held = kRopeHeld / ((int64_t)r.H * r.D / W) > 0 ? kRopeHeld / ((int64_t)r.H * r.D / W) : 1;
    r.nodes = (int32_t)std::min(std::min(even, most), held);
    const int64_t blocks = std::min<int64_t>((r.N + r.nodes - 1) / r.nodes, 8 * device_cus(dev));
    hipLaunchKernelGGL((gt_rope_kernel<T, W, PAIRS>), dim3((unsigned)blocks), dim3(kBlock), 0, stream, r);
    const hipError_t he = hipGetLastError();
    return he == hipSuccess ? GT_SUCCESS : hip_fail(he, "rotary launch");
}

// Units of fewer elements than this leave their rows to gt_rope_rows_kernel.
constexpr int kRopeRowsBelow = 4;

template <typename T>
gt_status launch_rope_rows(RopeParams r, int dev, hipStream_t stream) {
    const int64_t most = kRopeTable / (r.turned / 2), even = (r.N + 4 * device_cus(dev) - 1) / (4 * device_cus(dev));
    const int64_t held = kRopeHeld / r.H;  // (node and head rows below 2^16)
    r.nodes = (int32_t)std::min(std::min(even, most), held);
    const int64_t blocks = std::min<int64_t>((r.N + r.nodes - 1) / r.nodes, 8 * device_cus(dev));
    hipLaunchKernelGGL(gt_rope_rows_kernel<T>, dim3((unsigned)blocks), dim3(kBlock), 0, stream, r);
    const hipError_t he = hipGetLastError();
    return he == hipSuccess ? GT_SUCCESS : hip_fail(he, "rotary launch");
}

template <typename T>
gt_status pick_rope(const RopeParams& r, int dev, hipStream_t stream) {
    constexpr int kMost = 16 / Elt<T>::kBytes;
    const int w = rope_access(r, Elt<T>::kBytes);
    if (w < kRopeRowsBelow && r.D % kMost == 0) return launch_rope_rows<T>(r, dev, stream);
    if (r.layout == GT_ROPE_PAIRS) {  // (w is even: so are the sections)
        if constexpr (kMost == 8)
            if (w == 8) return launch_rope<T, 8, true>(r, dev, stream);
        if (w == 4) return launch_rope<T, 4, true>(r, dev, stream);
        return launch_rope<T, 2, true>(r, dev, stream);
    }
    if constexpr (kMost == 8)
        if (w == 8) return launch_rope<T, 8, false>(r, dev, stream);
    if (w == 4) return launch_rope<T, 4, false>(r, dev, stream);
    if (w == 2) return launch_rope<T, 2, false>(r, dev, stream);
    return launch_rope<T, 1, false>(r, dev, stream);
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
    r.copies = r.turned < D && (outQ != Q || outK != K);
    return dtype == GT_DTYPE_F32 ? pick_rope<float>(r, dev, stream) : pick_rope<bf16_tag>(r, dev, stream);
}
