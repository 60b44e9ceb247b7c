// Differential attention over a CSR graph, forward and backward (included by
// gt_attn.hip inside its anonymous namespace; on the row work order of
// gt_rows.hpp).  A value head h has two softmax maps over the row's entries,
// m = 0, 1, with query and key heads 2h + m of D elements, and values of 2D:
//     s_m,e = scale <Q_i,2h+m, K_j,2h+m>,  a_m = softmax of s_m over the row
//     out_i,h = sum_e (a_0,e - lambda_h a_1,e) V_j,h
// Q, K, V and out rows have the same 2HD elements.  A slice is PS whole pairs of
// maps.  A lane holds 16 bytes of a row: of one map's D elements in Q and K, and
// of the pair's 2D elements in V and out.  So a score is summed over the HL lanes
// of its map, and each lane then needs both maps' weights for its value elements:
// it computes its own map's and takes the other's from the lanes HL away.  The
// normalisers are known only at a row's end, hence two accumulators per element.
//
// Like the other row kernels these gather two random rows per entry and are bound
// by the path from L2 to the fabric (kernel time; bytes beyond the L2): forward,
// power law of 169 K nodes fp32 2x32 150 us, 7.1 TB/s; R-MAT of 1 M nodes bf16
// 2x32 1130 us, 6.7 TB/s, with the vector units busy for two thirds of it;
// lognormal 200 K nodes bf16 4x64 1600 us, 7.8 TB/s asked for; backward, R-MAT of
// 500 K nodes bf16 2x32 544 and 665 us, 6.3 and 6.5 TB/s.  Eight entries per step
// where a wavefront holds four groups (four / eight, us): 1130 / 1180, 544 / 581,
// 665 / 780.  All coefficients stay in fp32 and multiply exactly widened rows: the
// one rounding to bf16 is that of the results.

// The other map's value, from the other HL lanes of the pair (every lane of a
// map holds the same value).
template <int HL> __device__ __forceinline__ float pair_swap(float x) {
    static_assert(HL == 4 || HL == 8 || HL == 16 || HL == 32, "lanes of a map");
    if constexpr (HL == 4) return dpp<0x141>(x);  // row_half_mirror: other quad of 8
    if constexpr (HL == 8) return dpp<0x140>(x);  // row_mirror: other half of 16
    return __shfl_xor(x, HL);
}

struct DiffParams {
    RowWork w;
    // forward: Q, K, V, out; backward pass 0 (CSR rows): Q, dout | K, V; pass 1
    // (transposed rows): K, V | Q, dout
    const char* A;
    const char* B;
    const char* X;
    const char* Y;
    const float* lambda;  // [H]
    const float* lse;     // [N][2H] natural log (backward)
    float* lse_out;       // forward, or nullptr
    float2* stat;         // [N][2H] (lse log2(e), Delta): written by pass 0, read by pass 1
    char* out1;           // out, dQ or dK
    char* out2;           // dV
    float c;      // scale * log2(e)
    float scale;
    int32_t row_shift;
    int32_t maps;    // 2H
    int32_t slice0;  // slice of blockIdx.y == 0
    float* part;     // [slice of this launch][slot][kSlotFloats]
    int32_t* zero;   // a counter that the kernel without a partition clears, or nullptr
};

// What the lanes share while a wavefront works on one slice: base pointers at
// the slice's first element.
template <typename T, int PS, int D, bool BACKWARD>
struct DiffSlice {
    using Gm = Geo<T, 2 * PS, D>;
    static_assert(Gm::kNV == 1, "a slice is one 16-byte vector per lane");
    static constexpr int kG = Gm::kG, kHL = Gm::kHL, kEPV = Gm::kEPV;
    // Entries per step: four, whose registers leave room for more wavefronts; eight in
    // the forward where a row takes a whole wavefront (eight / four, us: R-MAT of 200 K
    // nodes, forward bf16 1x128 424 / 389, fp32 2x64 707 / 636, fp32 1x128 699 / 730,
    // backward 1178 / 933, 1645 / 1483, 1627 / 1607; lognormal 60 K nodes 202 / 205, 344 /
    // 350, 389 / 400, backward 413 / 399, 716 / 726, 757 / 778).
    static constexpr int kU = Gm::kU >= 8 && (BACKWARD || Gm::kP >= 2) ? 4 : Gm::kU;
    // Light rows in step order where a wavefront holds two rows or more (id order / so, us:
    // R-MAT of 200 K nodes, forward bf16 1x128 384 / 328, fp32 2x64 636 / 585, backward 930 /
    // 779, 1486 / 1355; degree 31 throughout the same).
    static constexpr bool kSorted = Gm::kP >= 2;
    static constexpr bool kDot2 = std::is_same<T, bf16_tag>::value;
    const char* A;
    const char* B;
    const char* X;
    const char* Y;
    const float* lambda;
    const float* lse;
    float* lse_out;
    float2* stat;
    char* out1;
    char* out2;
    float* part;
    float c, scale;
    int row_shift, maps;

    __device__ __forceinline__ uint64_t offset(int32_t row, int lig) const {
        return ((uint64_t)(uint32_t)row << row_shift) + (uint32_t)lig * 16u;
    }
    __device__ __forceinline__ static bool second(int lig) { return (lig / kHL) & 1; }
    __device__ __forceinline__ static int map(int lig) { return lig / kHL; }

    // Dot product of two rows' 16 bytes in this lane.
    __device__ __forceinline__ static float dot(const uint4& x, const uint4& y) {
        if constexpr (kDot2) {
            return dot8_bf16(x, y);
        } else {
            float a[kEPV], b[kEPV], d = 0.0f;
            widen<T>(x, a);
            widen<T>(y, b);
#pragma unroll
            for (int e = 0; e < kEPV; ++e) d = fmaf(a[e], b[e], d);
            return d;
        }
    }
};

template <typename Op, typename T, int PS, int D>
__device__ __forceinline__ Op diff_op(const DiffParams& p) {
    Op op;
    const int map = (p.slice0 + (int)blockIdx.y) * 2 * PS;
    const int64_t at = (int64_t)map * D * Elt<T>::kBytes;
    op.A = p.A + at;
    op.B = p.B + at;
    op.X = p.X + at;
    op.Y = p.Y + at;
    op.lambda = p.lambda + map / 2;
    op.lse = p.lse + map;
    op.lse_out = p.lse_out ? p.lse_out + map : nullptr;
    op.stat = p.stat + map;
    op.out1 = p.out1 + at;
    op.out2 = p.out2 + at;
    op.part = p.part + (int64_t)blockIdx.y * p.w.cap_slots * Op::kSlotFloats;
    op.c = p.c;
    op.scale = p.scale;
    op.row_shift = p.row_shift;
    op.maps = p.maps;
    return op;
}

// ------------------------------------------------------------------- forward

template <typename T, int PS, int D>
struct DiffFwdState;

template <typename T, int PS, int D>
struct DiffFwdOp : DiffSlice<T, PS, D, false> {
    using State = DiffFwdState<T, PS, D>;
    static constexpr int kRow = 2 * PS * D;
    static constexpr int kSlotFloats = 2 * kRow + 4 * PS;  // two accumulators, (max, sum) of each map
};

template <typename T, int PS, int D>
struct DiffFwdState {
    using Op = DiffFwdOp<T, PS, D>;
    static constexpr int EPV = Op::kEPV, kU = Op::kU, HL = Op::kHL;
    uint4 q;
    float own[EPV], other[EPV];  // sums by the weights of this lane's map, and of the pair's other map
    float m, l;                  // running max (log2 units) and sum of this lane's map

    __device__ __forceinline__ void reset() {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int e = 0; e < EPV; ++e) own[e] = other[e] = 0.0f;
    }

    __device__ __forceinline__ void begin(const Op& op, int32_t row, int lig) { q = load_once(op.A + op.offset(row, lig)); }

    struct Batch {
        uint4 k[kU], v[kU];
    };

    __device__ __forceinline__ void issue(const Op& op, const int32_t (&j)[kU], int lig, Batch& bt) const {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const uint64_t off = op.offset(j[u], lig);
            bt.k[u] = *reinterpret_cast<const uint4*>(op.X + off);
            bt.v[u] = *reinterpret_cast<const uint4*>(op.Y + off);
        }
    }

    __device__ __forceinline__ void consume(const Op& op, const Batch& bt, const int32_t (&)[kU], int nvalid) {
        // (no implicit contraction: the largest score's weight has to be exactly 1)
#pragma clang fp contract(off)
        float s[kU], mb = m;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const float d = head_sum<HL>(Op::dot(q, bt.k[u])) * op.c;  // unconditional: the sum is cross-lane
            s[u] = u < nvalid ? d : -INFINITY;
            mb = fmaxf(mb, s[u]);
        }
        // (while every score is -inf the weights are 0, not 2^(inf - inf))
        const float ref = mb == -INFINITY ? 0.0f : mb;
        const float corr = fast_exp2(m - ref), corr_x = pair_swap<HL>(corr);
        l *= corr;
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            own[e] *= corr;
            other[e] *= corr_x;
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const float p = fast_exp2(s[u] - ref), px = pair_swap<HL>(p);
            l += p;
            float v[EPV];
            widen<T>(bt.v[u], v);
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                own[e] = fmaf(p, v[e], own[e]);
                other[e] = fmaf(px, v[e], other[e]);
            }
        }
        m = mb;
    }

    // Merge the state of other entries of the same row.
    __device__ __forceinline__ void merge(float mo, float lo, const float (&oo)[EPV], const float (&xo)[EPV]) {
#pragma clang fp contract(off)
        const float mn = fmaxf(m, mo);
        const float ca = m == mn ? 1.0f : fast_exp2(m - mn), cb = mo == mn ? 1.0f : fast_exp2(mo - mn);
        const float cax = pair_swap<HL>(ca), cbx = pair_swap<HL>(cb);
        l = l * ca + lo * cb;
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            own[e] = own[e] * ca + oo[e] * cb;
            other[e] = other[e] * cax + xo[e] * cbx;
        }
        m = mn;
    }

    __device__ __forceinline__ void merge_xor(int off) {
        float oo[EPV], xo[EPV];
        const float mo = __shfl_xor(m, off), lo = __shfl_xor(l, off);
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            oo[e] = __shfl_xor(own[e], off);
            xo[e] = __shfl_xor(other[e], off);
        }
        merge(mo, lo, oo, xo);
    }

    __device__ __forceinline__ void store_out(const Op& op, int32_t row, int lig) const {
        const float inv = l > 0.0f ? 1.0f / l : l, inv_x = pair_swap<HL>(inv);  // (l NaN: NaN)
        const float lam = op.lambda[Op::map(lig) / 2];
        const bool second = Op::second(lig);
        float o[EPV];
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            const float a = own[e] * inv, b = other[e] * inv_x;
            o[e] = second ? fmaf(-lam, a, b) : fmaf(-lam, b, a);
        }
        store_once(op.out1 + op.offset(row, lig), narrow<T>(o));
        if (op.lse_out && lig % HL == 0) op.lse_out[(int64_t)row * op.maps + Op::map(lig)] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    }

    __device__ __forceinline__ void store_partial(const Op& op, int32_t slot, int lig) const {
        float* dst = op.part + (int64_t)slot * Op::kSlotFloats;
#pragma unroll
        for (int e = 0; e < EPV; e += 4) {
            *reinterpret_cast<float4*>(dst + lig * EPV + e) = make_float4(own[e], own[e + 1], own[e + 2], own[e + 3]);
            *reinterpret_cast<float4*>(dst + Op::kRow + lig * EPV + e) = make_float4(other[e], other[e + 1], other[e + 2], other[e + 3]);
        }
        if (lig % HL == 0) *reinterpret_cast<float2*>(dst + 2 * Op::kRow + 2 * Op::map(lig)) = make_float2(m, l);
    }

    struct Partial {
        float own[EPV], other[EPV];
        float2 ml;
    };

    __device__ __forceinline__ static void load_partial(const Op& op, int32_t slot, int lig, Partial& pt) {
        const float* src = op.part + (int64_t)slot * Op::kSlotFloats;
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            pt.own[e] = src[lig * EPV + e];
            pt.other[e] = src[Op::kRow + lig * EPV + e];
        }
        pt.ml = *reinterpret_cast<const float2*>(src + 2 * Op::kRow + 2 * Op::map(lig));
    }

    __device__ __forceinline__ void add(Partial& pt, bool valid) {
        if (!valid) {
            pt.ml = make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int e = 0; e < EPV; ++e) pt.own[e] = pt.other[e] = 0.0f;
        }
        merge(pt.ml.x, pt.ml.y, pt.own, pt.other);
    }
};

// ------------------------------------------------------------------ backward
//
// With a_m,e = exp(s_m,e - lse_m), c_e = <dO_i, V_j>, Delta_m = sum_e a_m,e c_e,
// g_0 = 1, g_1 = -lambda:
//     ds_m,e = g_m a_m,e (c_e - Delta_m)
//     dQ_m = scale sum ds_m K_m                          (pass 0, CSR rows)
//     dK_m = scale sum ds_m Q_m, dV = sum (a_0 - lambda a_1) dO   (pass 1, transposed rows)
//     dlambda = - sum over rows of Delta_1
// The forward's out gives only Delta_0 - lambda Delta_1, so pass 0 finds Delta
// itself in its one pass: with any c0 and t_e = a_e (c_e - c0),
//     sum a (c - Delta) K = sum t K - (sum t) sum a K,   Delta = c0 + sum t
// (sum a = 1).  c0 is the weighted mean of the c_e so far, so that nothing large
// cancels: a step moves the sums to the new mean c0' first (sum t grows by
// (c0 - c0') sum a, sum t K by (c0 - c0') sum a K), and so does a merge of two
// states.  A row of one entry gets exactly 0.

template <typename T, int PS, int D, int MODE>
struct DiffBwdState;

template <typename T, int PS, int D, int MODE>
struct DiffBwdOp : DiffSlice<T, PS, D, true> {
    using State = DiffBwdState<T, PS, D, MODE>;
    static constexpr int kRow = 2 * PS * D;
    static constexpr int kSlotFloats = 2 * kRow + (MODE == 0 ? 4 * 2 * PS : 0);
};

template <typename T, int PS, int D, int MODE>
struct DiffBwdState {
    using Op = DiffBwdOp<T, PS, D, MODE>;
    static constexpr int EPV = Op::kEPV, kU = Op::kU, HL = Op::kHL;
    uint4 a, b;                 // the row's own vectors
    float acc1[EPV], acc2[EPV];  // pass 0: sum t K, sum a K; pass 1: sum of ds Q, dV
    float L2;                   // pass 0: lse log2(e) of this lane's map
    float sum_t, sum_a, c0;     // pass 0
    float lam;                  // pass 1

    __device__ __forceinline__ void reset() {
        sum_t = sum_a = c0 = 0.0f;
#pragma unroll
        for (int e = 0; e < EPV; ++e) acc1[e] = acc2[e] = 0.0f;
    }

    // lse log2(e), with +inf for an empty map: its entries' weights are 0
    __device__ __forceinline__ static float weight_ref(float l2) { return l2 == -INFINITY ? INFINITY : l2; }

    __device__ __forceinline__ void begin(const Op& op, int32_t row, int lig) {
        const uint64_t off = op.offset(row, lig);
        a = load_once(op.A + off);
        b = load_once(op.B + off);
        if constexpr (MODE == 0)
            L2 = op.lse[(int64_t)row * op.maps + Op::map(lig)] * 1.4426950408889634f;
        else
            lam = op.lambda[Op::map(lig) / 2];
    }

    struct Batch {
        uint4 x[kU], y[kU];
        float2 st[MODE ? kU : 1];
    };

    __device__ __forceinline__ void issue(const Op& op, const int32_t (&j)[kU], int lig, Batch& bt) const {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const uint64_t off = op.offset(j[u], lig);
            bt.x[u] = *reinterpret_cast<const uint4*>(op.X + off);
            bt.y[u] = *reinterpret_cast<const uint4*>(op.Y + off);
            if constexpr (MODE == 1) bt.st[u] = op.stat[(int64_t)j[u] * op.maps + Op::map(lig)];
        }
    }

    __device__ __forceinline__ void consume(const Op& op, const Batch& bt, const int32_t (&)[kU], int nvalid) {
#pragma clang fp contract(off)
        float w[kU], cd[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const float s = head_sum<HL>(Op::dot(a, bt.x[u])) * op.c;
            cd[u] = head_sum<2 * HL>(Op::dot(b, bt.y[u]));
            const float l2 = weight_ref(MODE == 1 ? bt.st[MODE ? u : 0].x : L2);
            w[u] = u < nvalid ? fast_exp2(s - l2) : 0.0f;
        }
        if constexpr (MODE == 0) {
            const float base = sum_a > 0.0f ? c0 : cd[0];
            float ws = 0.0f, ts = 0.0f;
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                ws += w[u];
                ts = fmaf(w[u], cd[u] - base, ts);
            }
            recentre(mean_of(base, ts, sum_a + ws));
            sum_a += ws;
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const float t = w[u] * (cd[u] - c0);
                sum_t += t;
                float x[EPV];
                widen<T>(bt.x[u], x);
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    acc1[e] = fmaf(t, x[e], acc1[e]);
                    acc2[e] = fmaf(w[u], x[e], acc2[e]);
                }
            }
        } else {
            const bool second = Op::second(threadIdx.x % Op::kG);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const float ds = w[u] * (cd[u] - bt.st[u].y), wx = pair_swap<HL>(w[u]);
                const float mix = second ? fmaf(-lam, w[u], wx) : fmaf(-lam, wx, w[u]);
                float x[EPV], y[EPV];
                widen<T>(bt.x[u], x);
                widen<T>(bt.y[u], y);
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    acc1[e] = fmaf(ds, x[e], acc1[e]);
                    acc2[e] = fmaf(mix, y[e], acc2[e]);
                }
            }
        }
    }

    // base + sum / weight.  (The reciprocal is an estimate, and c0 need be no more.)
    __device__ __forceinline__ static float mean_of(float base, float sum, float weight) {
        return weight > 0.0f ? fmaf(sum, __builtin_amdgcn_rcpf(weight), base) : base;
    }

    __device__ __forceinline__ void recentre(float c) {
        const float shift = sum_a > 0.0f ? c0 - c : 0.0f;
        sum_t = fmaf(shift, sum_a, sum_t);
#pragma unroll
        for (int e = 0; e < EPV; ++e) acc1[e] = fmaf(shift, acc2[e], acc1[e]);
        c0 = c;
    }

    // Add the state of other entries of the same row.
    __device__ __forceinline__ void merge(const float (&o1)[EPV], const float (&o2)[EPV], float to, float ao, float co) {
        float shift = 0.0f;
        if constexpr (MODE == 0) {
            const float base = sum_a > 0.0f ? c0 : co;
            recentre(ao > 0.0f ? mean_of(base, ao * (co - base), sum_a + ao) : base);
            shift = ao > 0.0f ? co - c0 : 0.0f;
            sum_t += fmaf(shift, ao, to);
            sum_a += ao;
        }
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            acc1[e] += MODE == 0 ? fmaf(shift, o2[e], o1[e]) : o1[e];
            acc2[e] += o2[e];
        }
    }

    __device__ __forceinline__ void merge_xor(int off) {
        float o1[EPV], o2[EPV], to = 0.0f, ao = 0.0f, co = 0.0f;
        if constexpr (MODE == 0) {
            to = __shfl_xor(sum_t, off);
            ao = __shfl_xor(sum_a, off);
            co = __shfl_xor(c0, off);
        }
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            o1[e] = __shfl_xor(acc1[e], off);
            o2[e] = __shfl_xor(acc2[e], off);
        }
        merge(o1, o2, to, ao, co);
    }

    __device__ __forceinline__ void store_out(const Op& op, int32_t row, int lig) const {
        const uint64_t off = op.offset(row, lig);
        const float lm = op.lambda[Op::map(lig) / 2];
        const float g = (Op::second(lig) ? -lm : 1.0f) * op.scale;
        float o[EPV];
#pragma unroll
        for (int e = 0; e < EPV; ++e) o[e] = (MODE == 0 ? fmaf(-sum_t, acc2[e], acc1[e]) : acc1[e]) * g;
        store_once(op.out1 + off, narrow<T>(o));
        if constexpr (MODE == 0) {
            if (lig % HL == 0) {
                const int64_t at = (int64_t)row * op.maps + Op::map(lig);
                const float l2 = op.lse[at] * 1.4426950408889634f;
                op.stat[at] = make_float2(l2, l2 == -INFINITY ? 0.0f : c0 + sum_t);
            }
        } else {
            store_once(op.out2 + off, narrow<T>(acc2));
        }
    }

    __device__ __forceinline__ void store_partial(const Op& op, int32_t slot, int lig) const {
        float* dst = op.part + (int64_t)slot * Op::kSlotFloats;
#pragma unroll
        for (int e = 0; e < EPV; e += 4) {
            *reinterpret_cast<float4*>(dst + lig * EPV + e) = make_float4(acc1[e], acc1[e + 1], acc1[e + 2], acc1[e + 3]);
            *reinterpret_cast<float4*>(dst + Op::kRow + lig * EPV + e) = make_float4(acc2[e], acc2[e + 1], acc2[e + 2], acc2[e + 3]);
        }
        if constexpr (MODE == 0)
            if (lig % HL == 0)
                *reinterpret_cast<float4*>(dst + 2 * Op::kRow + 4 * Op::map(lig)) = make_float4(sum_t, sum_a, c0, 0.0f);
    }

    struct Partial {
        float a1[EPV], a2[EPV];
        float4 t;
    };

    __device__ __forceinline__ static void load_partial(const Op& op, int32_t slot, int lig, Partial& pt) {
        const float* src = op.part + (int64_t)slot * Op::kSlotFloats;
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            pt.a1[e] = src[lig * EPV + e];
            pt.a2[e] = src[Op::kRow + lig * EPV + e];
        }
        pt.t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if constexpr (MODE == 0) pt.t = *reinterpret_cast<const float4*>(src + 2 * Op::kRow + 4 * Op::map(lig));
    }

    __device__ __forceinline__ void add(Partial& pt, bool valid) {
        if (!valid) {
            pt.t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int e = 0; e < EPV; ++e) pt.a1[e] = pt.a2[e] = 0.0f;
        }
        merge(pt.a1, pt.a2, pt.t.x, pt.t.y, pt.t.z);
    }
};

// -------------------------------------------------------------------- kernels

template <typename Op, typename T, int PS, int D>
__global__ void __launch_bounds__(kBlock) gt_diff_kernel(DiffParams p) {
    __shared__ __attribute__((aligned(16))) int32_t tiles[kWavesPerBlock][kWave / Op::kG * TileOf<Op::kG>::kEntries];
    row_loop(p.w, diff_op<Op, T, PS, D>(p), tiles[threadIdx.x / kWave]);
}

// The partial states of each cut row, merged in a fixed order as in
// gt_bwd_merge_kernel: one wavefront per row and slice.  (Two pieces of a lane
// group in flight; with four the states take 152 registers and a row's eight
// pieces half of them: R-MAT of 1 M nodes bf16 2x32 57 against 44 us.)
constexpr uint32_t kDiffMergePieces = 2;

template <typename Op, typename T, int PS, int D>
__global__ void __launch_bounds__(kBlock) gt_diff_merge_kernel(DiffParams p) {
    constexpr uint32_t G = Op::kG, P = kWave / G;
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t g = lane / G;
    const int lig = lane % G;
    if (ROWS_CNT(p.w.counters, ROWS_PIECES) == 0) return;  // no long rows
    const CutRows cut(p.w, lane);
    const uint32_t n = cut.count(), waves = gridDim.x * kWavesPerBlock;
    const Op op = diff_op<Op, T, PS, D>(p);
    for (uint32_t i = blockIdx.x * kWavesPerBlock + wv; i < n; i += waves) {
        uint32_t slot, nq;
        const int32_t row = cut.row(p.w, i, lane, slot, nq);
        typename Op::State st;
        st.reset();
        for (uint32_t q0 = 0; q0 < nq; q0 += P * kDiffMergePieces) {
            // (a group without a piece reads the row's last and leaves it out)
            typename Op::State::Partial pt[kDiffMergePieces];
#pragma unroll
            for (uint32_t u = 0; u < kDiffMergePieces; ++u) {
                const uint32_t q = q0 + u * P + g;
                st.load_partial(op, (int32_t)(slot + (q < nq ? q : nq - 1)), lig, pt[u]);
            }
#pragma unroll
            for (uint32_t u = 0; u < kDiffMergePieces; ++u) st.add(pt[u], q0 + u * P + g < nq);
        }
#pragma unroll
        for (int off = G; off < kWave; off <<= 1) st.merge_xor(off);
        if (g == 0) st.store_out(op, row, lig);
    }
}

// Small graphs, without a partition: a workgroup takes as many rows as it has
// lane groups, in id order.  A group reads a row of up to kDirectAlone entries by
// itself; longer ones are then read one after another by all groups of the
// workgroup, a share each, and merged in LDS in a fixed order.  One launch takes
// the place of three (clear and partition, rows, merge).  (Rows read alone up to 16
// / 32 / 64 entries, us: 1.5 K nodes of degree 31, forward 33 / 11.4 / 11.5,
// backward 64 / 40 / 28; 1.5 K R-MAT nodes, backward 62 / 55 / 61.)
constexpr uint32_t kDirectAlone = 48;

template <typename Op, typename T, int PS, int D>
__global__ void __launch_bounds__(kBlock) gt_diff_direct_kernel(DiffParams p) {
    constexpr int G = Op::kG, P = kWave / G, U = Op::kU;
    constexpr uint32_t kGroups = kWavesPerBlock * P;
    __shared__ __attribute__((aligned(16))) float parts[kWavesPerBlock * Op::kSlotFloats];
    __shared__ uint64_t long_rows[kWavesPerBlock];
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lig = lane % G;
    const uint32_t group = wv * P + lane / G;
    Op op = diff_op<Op, T, PS, D>(p);
    op.part = parts;
    auto entries = [&](typename Op::State& st, uint32_t begin, uint32_t end) {
        int32_t j[U];
#pragma unroll
        for (int u = 0; u < U; ++u) j[u] = p.w.colidx[begin + u < end ? begin + u : end - 1];
        for (uint32_t t = begin; t < end; t += U) {
            typename Op::State::Batch bt;
            st.issue(op, j, lig, bt);
            int32_t next[U];
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = p.w.colidx[t + U + u < end ? t + U + u : end - 1];
            st.consume(op, bt, j, end - t < (uint32_t)U ? (int)(end - t) : U);
#pragma unroll
            for (int u = 0; u < U; ++u) j[u] = next[u];
        }
    };

    if (p.zero && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.zero = 0;
    const int64_t row0 = (int64_t)blockIdx.x * kGroups, row = row0 + group;
    uint32_t begin = 0, end = 0;
    if (row < p.w.N) {
        begin = (uint32_t)p.w.rowptr[row];
        end = (uint32_t)p.w.rowptr[row + 1];
    }
    const bool alone = end - begin <= kDirectAlone;
    const uint64_t longs = __ballot(!alone && lig == 0);
    if (lane == 0) long_rows[wv] = longs;
    if (row < p.w.N && alone) {
        typename Op::State st;
        st.reset();
        st.begin(op, (int32_t)row, lig);
        if (end > begin) entries(st, begin, end);
        st.store_out(op, (int32_t)row, lig);
    }
    __syncthreads();
    for (int w = 0; w < kWavesPerBlock; ++w) {
        for (uint64_t left = long_rows[w]; left; left &= left - 1) {
            const int64_t r = row0 + w * P + __builtin_ctzll(left) / G;
            const uint32_t rb = (uint32_t)p.w.rowptr[r], deg = (uint32_t)p.w.rowptr[r + 1] - rb;
            const uint32_t b = rb + (uint32_t)((uint64_t)deg * group / kGroups), e = rb + (uint32_t)((uint64_t)deg * (group + 1) / kGroups);
            typename Op::State st;
            st.reset();
            st.begin(op, (int32_t)r, lig);
            if (e > b) entries(st, b, e);
#pragma unroll
            for (int off = G; off < kWave; off <<= 1) st.merge_xor(off);
            if (lane < G) st.store_partial(op, wv, lig);
            __syncthreads();
            if (wv == 0) {
                st.reset();
#pragma unroll
                for (int k = 0; k < kWavesPerBlock; ++k) {
                    typename Op::State::Partial pt;
                    st.load_partial(op, k, lig, pt);
                    st.add(pt, true);
                }
                if (lane < G) st.store_out(op, (int32_t)r, lig);
            }
            __syncthreads();
        }
    }
}

// dlambda[h] = - sum over rows of Delta_1, in 64 bits: partial sums per
// workgroup, which the last workgroup to finish adds, in a fixed order.
constexpr int kLambdaBlocks = 256;

__global__ void __launch_bounds__(kBlock) gt_diff_lambda_kernel(const float2* stat, int64_t N, int32_t H, double* part, int32_t* done,
                                                                float* dlambda) {
    __shared__ double sums[kBlock];
    __shared__ int last;
    const int h = threadIdx.x % H, r = threadIdx.x / H, per = kBlock / H;
    auto reduce = [&](double s) {  // over the threads of a head, to the first
        sums[threadIdx.x] = s;
        __syncthreads();
        for (int off = kBlock / 2; off >= H; off >>= 1) {
            if ((int)threadIdx.x < off) sums[threadIdx.x] += sums[threadIdx.x + off];
            __syncthreads();
        }
    };
    double s = 0.0;
    const int64_t step = (int64_t)gridDim.x * per;
#pragma unroll 4
    for (int64_t i = (int64_t)blockIdx.x * per + r; i < N; i += step) s -= stat[(i * H + h) * 2 + 1].y;
    reduce(s);
    if (gridDim.x == 1) {
        if ((int)threadIdx.x < H) dlambda[threadIdx.x] = (float)sums[threadIdx.x];
        return;
    }
    if ((int)threadIdx.x < H) {
        __hip_atomic_store(part + blockIdx.x * H + threadIdx.x, sums[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __threadfence();
    }
    __syncthreads();
    if (threadIdx.x == 0) last = __hip_atomic_fetch_add(done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    s = 0.0;
    for (int b = r; b < (int)gridDim.x; b += per) s += __hip_atomic_load(part + b * H + h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    reduce(s);
    if ((int)threadIdx.x < H) dlambda[threadIdx.x] = (float)sums[threadIdx.x];
}

// ---------------------------------------------------------------------- host

struct DiffArgs {
    const int64_t* rowptr;
    const int32_t* colidx;
    const int64_t* rowptr_t;  // backward
    const int32_t* colidx_t;
    const void* Q;
    const void* K;
    const void* V;
    const float* lambda;
    const void* dout;  // backward
    const float* lse;  // backward
    void* out;         // forward
    float* lse_out;
    void* dQ;
    void* dK;
    void* dV;
    float* dlambda;
    int64_t N, E;
    int32_t H, D;
    float scale;
};

template <typename Op, typename T, int PS, int D>
int diff_resident(int dev) {
    static std::atomic<int> cache[64];
    if (dev < 0 || dev >= 64) return 4 * 256;
    if (cache[dev] == 0) {
        int nb = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&nb, gt_diff_kernel<Op, T, PS, D>, kBlock, 0) != hipSuccess || nb <= 0) nb = 4;
        cache[dev] = nb * device_cus(dev);
    }
    return cache[dev];
}

// The row kernel and the merge of the cut rows, slice by slice, after the
// partition of the rows.
template <typename Op, typename T, int PS, int D>
gt_status launch_diff_rows(DiffParams dp, const RowRule& rule, const SlotPlan& sp, const RowGrid& rg, int dev, PhaseEvents* ph, hipStream_t stream) {
    hipError_t he = hipSuccess;
    dp.w.long_blocks = rg.long_blocks;
    dp.w.light_first = rg.light_first;
    const int merge_grid = merge_blocks(sp, rule, device_cus(dev)), slices = dp.maps / (2 * PS);
    for (int s = 0; s < slices; s += sp.slices) {
        dp.slice0 = s;
        hipLaunchKernelGGL((gt_diff_kernel<Op, T, PS, D>), dim3(rg.blocks, sp.slices), dim3(kBlock), 0, stream, dp);
        if ((he = hipGetLastError()) != hipSuccess) return hip_fail(he, "differential attention launch");
        if (ph && s + sp.slices >= slices) ph->mark(2, stream);
        hipLaunchKernelGGL((gt_diff_merge_kernel<Op, T, PS, D>), dim3(merge_grid, sp.slices), dim3(kBlock), 0, stream, dp);
        if ((he = hipGetLastError()) != hipSuccess) return hip_fail(he, "differential attention merge launch");
    }
    return GT_SUCCESS;
}

// Whether a call takes its rows without a partition: small graphs, as long as
// their hubs' chains stay shorter than the launches saved (with a partition /
// without, us per call: forward of 2 K nodes of degree 9 fp32 1x32 20 / 11, power
// law of 4 K nodes (27 K entries) 25.5 / 19.3, of 8 K nodes (64 K) 26 / 43, 1.5 K
// R-MAT nodes (36 K) 25 / 22; bf16 4x64, power law of 1.5 K nodes (8 K) 26 / 13, of
// 4 K nodes 34 / 39; backward: 49 / 38, 54 / 84, 50 / 55, 55 / 32, 65 / 72).
bool diff_direct(int64_t N, int64_t E, int64_t row_bytes, const gt_tuning* tu) {
    return !tu && N <= 4096 && E <= 32768 && E * row_bytes <= (int64_t(16) << 20);
}

template <typename Op, typename T, int PS, int D>
gt_status launch_diff_direct(const DiffParams& dp, hipStream_t stream) {
    constexpr int kGroups = kWavesPerBlock * (kWave / Op::kG);
    hipLaunchKernelGGL((gt_diff_direct_kernel<Op, T, PS, D>), dim3((unsigned)((dp.w.N + kGroups - 1) / kGroups), dp.maps / (2 * PS)), dim3(kBlock),
                       0, stream, dp);
    const hipError_t he = hipGetLastError();
    return he == hipSuccess ? GT_SUCCESS : hip_fail(he, "differential attention launch");
}

// Workspace: two counter sets | statistics | light rows | long rows | partial
// states | partial sums of dlambda.
struct DiffPlan {
    RowRule rule;
    SlotPlan slots;
    size_t o_stat, o_light, o_deg, o_long, o_part, o_lambda, bytes;
};

template <typename Op, int PS>
DiffPlan plan_diff(const DiffArgs& a, int gather_bytes, int slot_bytes, bool backward, const gt_tuning* tu) {
    DiffPlan p;
    const int slices = a.H / PS;
    p.rule = row_rule(a.N, a.E, slices, gather_bytes, backward ? 2 * slot_bytes + 1024 : 3 * (2 * slot_bytes + 256) / 4, Op::Gm::kP, tu);
    size_t off = align_up((2 * kRowsSetWords + kRowsStride) * sizeof(int32_t), 256);  // (and a counter)
    auto place = [&off](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return at;
    };
    p.o_stat = place(backward ? (size_t)a.N * a.H * 2 * sizeof(float2) : 0);
    p.o_light = place(Op::kSorted ? (size_t)a.N * sizeof(LightRow) : 0);
    p.o_deg = place(Op::kSorted ? (size_t)a.N : 0);
    p.o_long = place((size_t)long_list_rows(a.N, a.E, p.rule.light_max) * sizeof(LongRow));
    p.slots = slot_plan(p.rule, slices, slot_bytes, off, false);
    p.o_part = place((size_t)p.slots.cap * p.slots.slices * slot_bytes);
    p.o_lambda = place(backward ? (size_t)kLambdaBlocks * a.H * sizeof(double) : 0);
    p.bytes = off;
    return p;
}

template <typename Op>
void diff_work(RowWork& w, const DiffArgs& a, const DiffPlan& plan, char* ws) {
    w.rowptr = a.rowptr;
    w.colidx = a.colidx;
    w.N = a.N;
    w.E = (uint32_t)a.E;
    set_rule(w, plan.rule);
    w.cap_slots = plan.slots.cap;
    w.long_list = reinterpret_cast<LongRow*>(ws + plan.o_long);
    w.light_list = Op::kSorted ? reinterpret_cast<LightRow*>(ws + plan.o_light) : nullptr;
    w.light_deg = reinterpret_cast<uint8_t*>(ws + plan.o_deg);
    w.long_blocks = 0;
    w.light_first = false;
    w.maybe_no_light = false;
}

template <typename T, int PS, int D>
void diff_features(DiffParams& dp, const DiffArgs& a) {
    dp.lambda = a.lambda;
    dp.lse = a.lse;
    dp.c = a.scale * 1.4426950408889634f;
    dp.scale = a.scale;
    dp.row_shift = floor_log2((uint64_t)2 * a.H * a.D * Elt<T>::kBytes);
    dp.maps = 2 * a.H;
}

template <typename T, int PS, int D>
gt_status launch_diff_fwd(const DiffArgs& a, const gt_tuning* tu, hipStream_t stream) {
    using Op = DiffFwdOp<T, PS, D>;
    constexpr int kSlotBytes = Op::kSlotFloats * (int)sizeof(float);
    int dev = 0;
    if (const gt_status ds = call_device(stream, &dev); ds != GT_SUCCESS) return ds;
    hipError_t he = hipSuccess;
    DiffParams dp{};
    diff_features<T, PS, D>(dp, a);
    dp.A = static_cast<const char*>(a.Q);
    dp.B = dp.A;
    dp.X = static_cast<const char*>(a.K);
    dp.Y = static_cast<const char*>(a.V);
    dp.lse_out = a.lse_out;
    dp.out1 = static_cast<char*>(a.out);
    dp.out2 = dp.out1;
    PhaseEvents ph;
    if (diff_direct(a.N, a.E, (int64_t)2 * a.H * a.D * Elt<T>::kBytes, tu)) {
        dp.w.rowptr = a.rowptr;
        dp.w.colidx = a.colidx;
        dp.w.N = a.N;
        if ((he = ph.start(stream)) != hipSuccess) return hip_fail(he, "profiling events");
        ph.mark(1, stream);
        if (const gt_status st = launch_diff_direct<Op, T, PS, D>(dp, stream); st != GT_SUCCESS) return st;
        ph.mark(2, stream);
        ph.commit(stream);
        return GT_SUCCESS;
    }
    const DiffPlan plan = plan_diff<Op, PS>(a, 2 * Op::kRow * Elt<T>::kBytes, kSlotBytes, false, tu);
    const RowGrid rg = row_grid(a.N, a.E, Op::Gm::kP, plan.slots.slices, false, diff_resident<Op, T, PS, D>(dev), tu);
    CallWorkspace cw;
    gt_status st = acquire_workspace(dev, plan.bytes, stream, cw);
    if (st != GT_SUCCESS) return st;
    diff_work<Op>(dp.w, a, plan, cw.ptr);
    dp.part = reinterpret_cast<float*>(cw.ptr + plan.o_part);
    // counter sets as in the attention forward: a cached block alternates between
    // its two, and the partition clears the one of the block's next call
    int32_t* cnt = reinterpret_cast<int32_t*>(cw.ptr);
    const bool alternate = cw.kind == CallWorkspace::CACHED;
    dp.w.counters = cnt + (alternate ? (cw.block.gen & 1u) * kRowsSetWords : 0);
    if ((he = ph.start(stream)) != hipSuccess) return hip_fail(he, "profiling events");
    if (!(alternate && cw.block.primed) && (he = clear_counters(dp.w.counters, kRowsSetWords, stream)) != hipSuccess)
        return hip_fail(he, "counter clear");
    SortParams pp;
    pp.w = dp.w;
    pp.step = Op::kU;
    pp.groups = Op::Gm::kP;
    if (alternate) pp.zero_next = cnt + ((cw.block.gen + 1u) & 1u) * kRowsSetWords;
    if ((he = launch_sort_rows(pp, stream)) != hipSuccess) return hip_fail(he, "partition launch");
    if (alternate) {
        ++cw.block.gen;
        cw.keep_primed = true;
    }
    ph.mark(1, stream);
    st = launch_diff_rows<Op, T, PS, D>(dp, plan.rule, plan.slots, rg, dev, &ph, stream);
    if (st != GT_SUCCESS) return st;
    ph.commit(stream);
    return GT_SUCCESS;
}

template <typename T, int PS, int D, int MODE>
gt_status launch_diff_bwd_pass(DiffParams dp, const DiffArgs& a, const DiffPlan& plan, int dev, hipStream_t stream) {
    using Op = DiffBwdOp<T, PS, D, MODE>;
    const RowGrid rg = row_grid(a.N, a.E, Op::Gm::kP, plan.slots.slices, false, diff_resident<Op, T, PS, D>(dev), nullptr);
    SortParams pp;
    pp.w = dp.w;
    pp.step = Op::kU;
    pp.groups = Op::Gm::kP;
    if (const hipError_t he = launch_sort_rows(pp, stream); he != hipSuccess) return hip_fail(he, "partition launch");
    return launch_diff_rows<Op, T, PS, D>(dp, plan.rule, plan.slots, rg, dev, nullptr, stream);
}

template <typename T, int PS, int D>
gt_status launch_diff_bwd(const DiffArgs& a, const gt_tuning*, hipStream_t stream) {
    using Op = DiffBwdOp<T, PS, D, 0>;
    constexpr int kSlotBytes = Op::kSlotFloats * (int)sizeof(float);  // (pass 1: the accumulators alone)
    const bool direct = diff_direct(a.N, a.E, (int64_t)2 * a.H * a.D * Elt<T>::kBytes, nullptr);
    const DiffPlan plan = plan_diff<Op, PS>(a, 2 * Op::kRow * Elt<T>::kBytes, kSlotBytes, true, nullptr);
    int dev = 0;
    if (const gt_status ds = call_device(stream, &dev); ds != GT_SUCCESS) return ds;
    CallWorkspace cw;
    gt_status st = acquire_workspace(dev, plan.bytes, stream, cw);
    if (st != GT_SUCCESS) return st;
    int32_t* cnt = reinterpret_cast<int32_t*>(cw.ptr);
    int32_t* done = cnt + 2 * kRowsSetWords;
    hipError_t he = hipSuccess;
    const int64_t per = kBlock / a.H * 8;
    const int blocks = (int)(a.N / per + 1 < kLambdaBlocks ? a.N / per + 1 : kLambdaBlocks);
    if (!direct && (he = clear_counters(cnt, 2 * kRowsSetWords + kRowsStride, stream)) != hipSuccess)
        return hip_fail(he, "counter clear");
    DiffParams dp{};
    diff_work<Op>(dp.w, a, plan, cw.ptr);
    diff_features<T, PS, D>(dp, a);
    dp.stat = reinterpret_cast<float2*>(cw.ptr + plan.o_stat);
    dp.part = reinterpret_cast<float*>(cw.ptr + plan.o_part);
    dp.zero = done;
    for (int mode = 0; mode < 2; ++mode) {
        dp.w.rowptr = mode == 0 ? a.rowptr : a.rowptr_t;
        dp.w.colidx = mode == 0 ? a.colidx : a.colidx_t;
        dp.w.counters = cnt + mode * kRowsSetWords;
        dp.A = static_cast<const char*>(mode == 0 ? a.Q : a.K);
        dp.B = static_cast<const char*>(mode == 0 ? a.dout : a.V);
        dp.X = static_cast<const char*>(mode == 0 ? a.K : a.Q);
        dp.Y = static_cast<const char*>(mode == 0 ? a.V : a.dout);
        dp.out1 = static_cast<char*>(mode == 0 ? a.dQ : a.dK);
        dp.out2 = static_cast<char*>(a.dV);
        if (direct)
            st = mode == 0 ? launch_diff_direct<DiffBwdOp<T, PS, D, 0>, T, PS, D>(dp, stream)
                           : launch_diff_direct<DiffBwdOp<T, PS, D, 1>, T, PS, D>(dp, stream);
        else
            st = mode == 0 ? launch_diff_bwd_pass<T, PS, D, 0>(dp, a, plan, dev, stream)
                           : launch_diff_bwd_pass<T, PS, D, 1>(dp, a, plan, dev, stream);
        if (st != GT_SUCCESS) return st;
    }
    if (a.dlambda) {
        hipLaunchKernelGGL(gt_diff_lambda_kernel, dim3(blocks), dim3(kBlock), 0, stream, dp.stat, a.N, a.H,
                           reinterpret_cast<double*>(cw.ptr + plan.o_lambda), done, a.dlambda);
        if ((he = hipGetLastError()) != hipSuccess) return hip_fail(he, "lambda gradient launch");
    }
    return GT_SUCCESS;
}

using DiffFn = gt_status (*)(const DiffArgs&, const gt_tuning*, hipStream_t);

template <typename T, int PS, int D>
DiffFn diff_fn(bool backward) {
    return backward ? &launch_diff_bwd<T, PS, D> : &launch_diff_fwd<T, PS, D>;
}

// Slices: the pairs of 256 bytes, or one where a pair has more.
template <typename T>
DiffFn pick_diff(bool backward, int32_t H, int32_t D) {
    constexpr bool kBf16 = std::is_same<T, bf16_tag>::value;
    if (H != 1 && H != 2 && H != 4 && H != 8) return nullptr;
    switch (D) {
        case 32:
            if constexpr (kBf16)
                if (H >= 2) return diff_fn<T, 2, 32>(backward);
            return diff_fn<T, 1, 32>(backward);
        case 64: return diff_fn<T, 1, 64>(backward);
        case 128: return diff_fn<T, 1, 128>(backward);
        case 256:
            if constexpr (kBf16) return diff_fn<T, 1, 256>(backward);
            return nullptr;
        default: return nullptr;
    }
}

gt_status run_diff(gt_dtype dtype, const DiffArgs& a, bool backward, const gt_tuning* tu, hipStream_t stream) {
    t_last_error.clear();
    if (check_tuning(tu) != GT_SUCCESS) return GT_ERROR_INVALID_VALUE;
    if (dtype != GT_DTYPE_F32 && dtype != GT_DTYPE_BF16) return fail(GT_ERROR_NOT_SUPPORTED, "unknown dtype");
    if (a.N < 0 || a.N >= (int64_t(1) << 31)) return fail(GT_ERROR_INVALID_VALUE, "N must be in [0, 2^31)");
    if (a.E < 0 || a.E >= (int64_t(1) << 31)) return fail(GT_ERROR_INVALID_VALUE, "E must be in [0, 2^31)");
    if (a.H < 1 || a.D < 1) return fail(GT_ERROR_INVALID_VALUE, "H and D must be positive");
    if (!std::isfinite(a.scale)) return fail(GT_ERROR_INVALID_VALUE, "scale must be finite");
    const DiffFn fn = dtype == GT_DTYPE_F32 ? pick_diff<float>(backward, a.H, a.D) : pick_diff<bf16_tag>(backward, a.H, a.D);
    if (!fn)
        return fail(GT_ERROR_NOT_SUPPORTED, "unsupported (H, D) = (" + std::to_string(a.H) + ", " + std::to_string(a.D) +
                                                "); H in {1,2,4,8} with D in {32,64,128}, or bf16 D = 256");
    struct Buffer {
        const void* ptr;
        size_t bytes, align;
        const char* name;
    };
    const size_t rows = (size_t)a.N * 2 * a.H * a.D * (dtype == GT_DTYPE_F32 ? 4 : 2), maps = (size_t)a.N * 2 * a.H * sizeof(float),
                 heads = (size_t)a.H * sizeof(float);
    const Buffer dlam{a.dlambda, heads, 4, "dlambda"};
    if (a.N == 0) {
        if (!backward || !a.dlambda) return GT_SUCCESS;
        if (reinterpret_cast<uintptr_t>(a.dlambda) % 4 != 0) return fail(GT_ERROR_INVALID_VALUE, "dlambda must be 4-byte aligned");
        int dev = 0;
        if (const gt_status ds = call_device(stream, &dev); ds != GT_SUCCESS) return ds;
        const hipError_t he = clear_counters(reinterpret_cast<int32_t*>(a.dlambda), a.H, stream);  // (0.0f is all bits 0)
        return he == hipSuccess ? GT_SUCCESS : hip_fail(he, "lambda gradient launch");
    }
    if (!a.rowptr || (backward && !a.rowptr_t)) return fail(GT_ERROR_INVALID_VALUE, "rowptr or rowptr_t is null");
    if (a.E > 0 && (!a.colidx || (backward && !a.colidx_t))) return fail(GT_ERROR_INVALID_VALUE, "colidx or colidx_t is null");
    const Buffer fwd_ins[] = {{a.Q, rows, 16, "Q"}, {a.K, rows, 16, "K"}, {a.V, rows, 16, "V"}, {a.lambda, heads, 4, "lambda"}};
    const Buffer bwd_ins[] = {{a.Q, rows, 16, "Q"}, {a.K, rows, 16, "K"}, {a.V, rows, 16, "V"}, {a.lambda, heads, 4, "lambda"},
                              {a.dout, rows, 16, "dout"}, {a.lse, maps, 4, "lse"}};
    const Buffer fwd_outs[] = {{a.out, rows, 16, "out"}, {a.lse_out, maps, 4, "lse"}};
    const Buffer bwd_outs[] = {{a.dQ, rows, 16, "dQ"}, {a.dK, rows, 16, "dK"}, {a.dV, rows, 16, "dV"}, dlam};
    const Buffer* ins = backward ? bwd_ins : fwd_ins;
    const Buffer* outs = backward ? bwd_outs : fwd_outs;
    const int n_ins = backward ? 6 : 4, n_outs = backward ? 4 : 2;
    for (int k = 0; k < n_ins + n_outs; ++k) {
        const Buffer& b = k < n_ins ? ins[k] : outs[k - n_ins];
        const bool optional = k == n_ins + n_outs - 1;  // lse of the forward, dlambda
        if ((!b.ptr && !optional) || reinterpret_cast<uintptr_t>(b.ptr) % b.align != 0)
            return fail(GT_ERROR_INVALID_VALUE, std::string(b.name) + (optional ? " must be " : " must be non-null and ") + std::to_string(b.align) + "-byte aligned");
    }
    for (int k = 0; k < n_outs; ++k) {
        if (!outs[k].ptr) continue;
        for (int i = 0; i < n_ins + k; ++i) {
            const Buffer& b = i < n_ins ? ins[i] : outs[i - n_ins];
            if (b.ptr && overlaps(outs[k].ptr, outs[k].bytes, b.ptr, b.bytes))
                return fail(GT_ERROR_INVALID_VALUE, std::string(outs[k].name) + " overlaps " + b.name);
        }
    }
    return fn(a, tu, stream);
}
