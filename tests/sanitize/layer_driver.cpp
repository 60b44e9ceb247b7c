// Every entry point of include/gt_layer.h through its whole host side, over the
// stand-in runtime of hip_stub.cpp (kernels do not run): shapes on each side of
// every choice of a kernel, empty graphs, optional buffers.  Prints the failures.
#include <cstdio>
#include <vector>

#include "gt_layer.h"

static int failures = 0;
static void expect(gt_status got, gt_status want, const char* what) {
    if (got == want) return;
    ++failures;
    std::printf("%s: status %d, wanted %d (%s)\n", what, (int)got, (int)want, gt_last_error_message());
}

int main() {
    auto buf = [](size_t n) {
        void* p = nullptr;
        (void)hipMalloc(&p, n);
        return p;
    };
    std::vector<void*> held;
    auto get = [&](size_t n) {
        held.push_back(buf(n + 64));
        return held.back();
    };
    for (int dt = 0; dt < 2; ++dt) {
        const gt_dtype t = (gt_dtype)dt;
        const size_t eb = dt ? 2 : 4;
        for (int64_t N : {1, 300, 5000, 70000})
            for (int H : {1, 2, 4, 8})
                for (int D : {32, 64, 128, 256}) {
                    if (D == 256 && !dt) continue;
                    const int64_t E = N * 9;
                    const size_t row = (size_t)N * 2 * H * D * eb;
                    if (row > (size_t(64) << 20)) continue;
                    auto* rp = (int64_t*)get((N + 1) * 8);
                    auto* ci = (int32_t*)get(E * 4);
                    void *q = get(row), *k = get(row), *v = get(row), *o = get(row), *dq = get(row), *dk = get(row), *dv = get(row), *dout = get(row);
                    auto *lam = (float*)get(H * 4), *dl = (float*)get(H * 4), *lse = (float*)get((size_t)N * 2 * H * 4);
                    const gt_tuning tu = {2, 6, 64, 0, 0, 0};
                    expect(gt_diff_attn_fwd(t, rp, ci, q, k, v, lam, o, lse, N, E, H, D, 0.1f, nullptr, nullptr), GT_SUCCESS, "diff forward");
                    expect(gt_diff_attn_fwd(t, rp, ci, q, k, v, lam, o, nullptr, N, E, H, D, 0.1f, &tu, nullptr), GT_SUCCESS, "diff forward, tuned");
                    expect(gt_diff_attn_fwd(t, rp, nullptr, q, k, v, lam, o, nullptr, N, 0, H, D, 0.1f, nullptr, nullptr), GT_SUCCESS, "diff forward, no entries");
                    expect(gt_diff_attn_bwd(t, rp, ci, rp, ci, q, k, v, lam, dout, lse, dq, dk, dv, dl, N, E, H, D, 0.1f, nullptr), GT_SUCCESS, "diff backward");
                    expect(gt_diff_attn_bwd(t, rp, ci, rp, ci, q, k, v, lam, dout, lse, dq, dk, dv, nullptr, N, E, H, D, 0.1f, nullptr), GT_SUCCESS, "diff backward, no dlambda");
                    expect(gt_diff_attn_bwd(t, rp, ci, rp, ci, q, k, v, lam, dout, lse, q, dk, dv, dl, N, E, H, D, 0.1f, nullptr), GT_ERROR_INVALID_VALUE, "diff backward, aliased");
                    for (void* p : held) (void)hipFree(p);
                    held.clear();
                }
        for (int layout = 0; layout < 3; ++layout)
            for (int64_t N : {1, 4097, 100000}) {
                const int shapes[][6] = {{1, 2, 2, 0, 0, 0}, {8, 64, 16, 24, 24, 0}, {3, 40, 4, 2, 10, 0}, {2, 512, 128, 128, 128, 128}, {4, 32, 32, 0, 0, 0}};
                for (const auto& s : shapes) {
                    gt_rope_spec spec = {0, {0, 0, 0, 0}, layout, 1e4};
                    for (int a = 0; a < 4 && s[2 + a]; ++a) spec.dims[spec.axes++] = s[2 + a];
                    const size_t bytes = (size_t)N * s[0] * s[1] * eb;
                    if (bytes > (size_t(64) << 20)) continue;
                    auto* pos = (float*)get((size_t)N * spec.axes * 4);
                    void *q = get(bytes), *k = get(bytes), *oq = get(bytes);
                    expect(gt_rope(t, pos, q, k, oq, k, N, s[0], s[1], &spec, 0, nullptr), GT_SUCCESS, "rope");
                    expect(gt_rope(t, pos, q, nullptr, q, nullptr, N, s[0], s[1], &spec, 1, nullptr), GT_SUCCESS, "rope in place");
                    for (void* p : held) (void)hipFree(p);
                    held.clear();
                }
            }
        for (int64_t N : {1, 257, 20000})
            for (int F : {1, 7, 64, 203, 512, 1000, 1024, 2048, 2049, 4097, 8192, 12345, 16383, 16384}) {
                const size_t bytes = (size_t)N * F * eb;
                if (bytes > (size_t(128) << 20)) continue;
                void *x = get(bytes), *dy = get(bytes), *y = get(bytes);
                auto *g = (float*)get(F * 4), *b = (float*)get(F * 4), *dg = (float*)get(F * 4), *db = (float*)get(F * 4), *m = (float*)get(N * 4), *r = (float*)get(N * 4);
                expect(gt_layernorm_fwd(t, x, g, b, y, m, r, N, F, 1e-5f, nullptr), GT_SUCCESS, "norm forward");
                expect(gt_layernorm_fwd(t, x, nullptr, nullptr, x, nullptr, nullptr, N, F, 0.0f, nullptr), GT_SUCCESS, "norm forward in place");
                expect(gt_layernorm_bwd(t, x, dy, g, m, r, y, dg, db, N, F, nullptr), GT_SUCCESS, "norm backward");
                expect(gt_layernorm_bwd(t, x, dy, nullptr, m, r, dy, nullptr, db, N, F, nullptr), GT_SUCCESS, "norm backward in place");
                expect(gt_layernorm_bwd(t, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, dg, db, 0, F, nullptr), GT_SUCCESS, "norm backward, no rows");
                for (void* p : held) (void)hipFree(p);
                held.clear();
            }
    }
    (void)gt_workspace_release();
    std::printf("%d failure(s)\n", failures);
    return failures ? 1 : 0;
}
