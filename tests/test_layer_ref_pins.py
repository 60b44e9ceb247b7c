"""The plain float64 forms that the GPU tests compare with (tests/layer_ref.py),
pinned on the CPU: gradients against differences of the forward, the inverse
rotation, and hand-computed values."""
import math

import numpy as np
import pytest

import synth
from tests import layer_ref as ref


def small(seed, H=2, D=32, N=30):
    rowptr, colidx = synth.ragged_graph(seed, N, max_deg=6, empty_frac=0.2, hubs={3: 25}, self_loops=False, shuffle=True)
    Q, K, V = synth.features(seed, N, 2 * H, D, "f32")
    lam = np.linspace(-0.5, 0.9, H).astype(np.float32)
    return rowptr, colidx, Q, K, V.reshape(N, H, 2 * D), lam


def test_diff_gradients_against_differences():
    rowptr, colidx, Q, K, V, lam = small(1)
    dO = synth.features(2, *V.shape, "f32")[0]
    r = ref.Diff(rowptr, colidx, Q, K, V, lam, 0.2, dO)
    rng = np.random.default_rng(0)
    names = {"Q": r.dQ, "K": r.dK, "V": r.dV, "lam": r.dlam}
    for name, grad in names.items():
        step = rng.standard_normal(grad.shape)
        vals = []
        for sign in (1, -1):
            x = {"Q": Q, "K": K, "V": V, "lam": lam}
            x[name] = x[name].astype(np.float64) + sign * 1e-5 * step
            vals.append(float(np.sum(ref.Diff(rowptr, colidx, x["Q"], x["K"], x["V"], x["lam"], 0.2).out * dO)))
        # (the second difference's error is of order 1e-10 of the value)
        assert abs((vals[0] - vals[1]) / 2e-5 - float(np.sum(grad * step))) < 1e-5 * (1 + float(np.sum(np.abs(grad * step)))), name


def test_diff_by_hand():
    # two entries: weights 1/2, 1/2 in the first map and 3/4, 1/4 in the second
    rowptr, colidx = np.array([0, 2, 2], np.int64), np.array([0, 1], np.int32)
    Q, K = np.zeros((2, 2, 32), np.float32), np.zeros((2, 2, 32), np.float32)
    Q[0, 1, 0], K[0, 1, 0] = 1.0, math.log(3.0)
    V = np.zeros((2, 1, 64), np.float32)
    V[0], V[1] = 1.0, 5.0
    r = ref.Diff(rowptr, colidx, Q, K, V, np.array([0.5], np.float32), 1.0)
    assert np.allclose(r.out[0], 0.5 * 1 + 0.5 * 5 - 0.5 * (0.75 * 1 + 0.25 * 5), rtol=1e-7)
    assert np.all(r.out[1] == 0) and np.all(np.isneginf(r.lse[1]))
    assert np.allclose(r.lse[0], [math.log(2), math.log(4)])


def test_norm_gradients_against_differences():
    rng = np.random.default_rng(3)
    X, dO = rng.standard_normal((7, 13)) + 2, rng.standard_normal((7, 13))
    gamma, beta = rng.standard_normal(13), rng.standard_normal(13)
    r0 = ref.Norm(X, gamma, beta, 1e-3)
    r = ref.Norm(X, gamma, beta, 1e-3, dO, r0.mean, r0.rstd)
    for name, grad in {"X": r.dX, "gamma": r.dgamma, "beta": r.dbeta}.items():
        step, vals = rng.standard_normal(grad.shape), []
        for sign in (1, -1):
            x = {"X": X, "gamma": gamma, "beta": beta}
            x[name] = x[name] + sign * 1e-5 * step
            vals.append(float(np.sum(ref.Norm(x["X"], x["gamma"], x["beta"], 1e-3).out * dO)))
        assert abs((vals[0] - vals[1]) / 2e-5 - float(np.sum(grad * step))) < 1e-6 * (1 + float(np.sum(np.abs(grad * step)))), name


@pytest.mark.parametrize("layout", ["pairs", "halves", "sections"])
def test_rope_turns_and_turns_back(layout):
    rng = np.random.default_rng(5)
    pos, x = rng.uniform(-50, 50, (9, 3)).astype(np.float32), rng.standard_normal((9, 2, 32))
    y, _ = ref.rope(pos, x, [6, 12, 10], 100.0, layout, False)
    z, _ = ref.rope(pos, y, [6, 12, 10], 100.0, layout, True)
    assert np.allclose(z, x, atol=1e-12) and not np.allclose(y, x, atol=0.1)
    assert np.allclose(np.sum(y ** 2, -1), np.sum(x ** 2, -1)) and np.array_equal(y[..., 28:], x[..., 28:])
    # products of a query and a key depend on the difference of their positions alone
    k = rng.standard_normal(x.shape)
    far, _ = ref.rope(pos + np.float32(16), x, [6, 12, 10], 100.0, layout, False)
    near = np.sum(y * ref.rope(pos - np.float32(16), k, [6, 12, 10], 100.0, layout, False)[0], -1)
    assert np.allclose(np.sum(far * ref.rope(pos, k, [6, 12, 10], 100.0, layout, False)[0], -1), near, atol=1e-4)


def test_rope_by_hand():
    # position pi / 2 at the first frequency, 1: (x, y) -> (-y, x); the second pair by 100^-1/2 of that
    pos = np.array([[math.pi / 2]], np.float32)
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    y, _ = ref.rope(pos, x, [4], 100.0, "pairs", False)
    a = math.pi / 20
    want = [-2, 1, 3 * math.cos(a) - 4 * math.sin(a), 3 * math.sin(a) + 4 * math.cos(a)]
    assert np.allclose(y[0, 0], want, atol=1e-6)
    y, _ = ref.rope(pos, x[..., [0, 2, 1, 3]], [4], 100.0, "halves", False)
    assert np.allclose(y[0, 0][[0, 2, 1, 3]], want, atol=1e-6)


def test_bench_byte_models():
    import bench
    # every gathered row of 2HD elements charged; the others read and written once
    assert bench.layer_model_bytes("diff", 10, 40, 4, 32, 4) == 8 * 11 + 4 * 40 + 2 * 10 * 512 + 2 * 40 * 512
    assert bench.layer_model_bytes("rope", 10, 40, 4, 32, 2) == 40 + 4 * 10 * 256
    assert bench.layer_model_bytes("layernorm", 10, 40, 4, 32, 2) == 2 * 10 * 256 + 80 + 8 * 128
