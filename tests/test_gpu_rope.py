"""Rotary positions with several axes on the GPU, through the C ABI against the
float64 form of tests/layer_ref.py.

Tolerance: the angle is reduced in 64 bits, its sine and cosine are held to
2^-21 (the reduced angle's rounding to fp32 and the functions' own error), so
an element is off by at most (|x| + |y|) (2^-21 + 2^-23) and one rounding."""
import numpy as np
import pytest

import synth
from tests import layer_ref as ref
from tests.helpers import to_device, to_host_f32

pytestmark = pytest.mark.gpu

TRIG = 2.0 ** -21 + 2.0 ** -23


def run(pos, Q, dims, K=None, theta=10000.0, layout="pairs", inverse=False, in_place=False):
    import torch
    import paper_2605_31500_amd as gt
    p, q = to_device(pos), to_device(Q)
    k = None if K is None else to_device(K)
    oq = q if in_place else torch.full_like(q, float("nan"))
    ok = None if K is None else k if in_place else torch.full_like(k, float("nan"))
    gt.gt_rope(p, q, oq, dims, K=k, out_k=ok, theta=theta, layout=layout, inverse=inverse)
    torch.cuda.synchronize()
    return to_host_f32(oq), None if K is None else to_host_f32(ok)


def check(got, pos, X, dims, theta, layout, inverse, dtype):
    want, size = ref.rope(pos, X, dims, theta, layout, inverse)
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - want) <= TRIG * size + ref.ROUND[dtype] * (np.abs(want) + TRIG * size))


def positions(seed, N, axes, kind):
    rng = np.random.default_rng(seed)
    if kind == "grid":
        return np.stack(np.unravel_index(np.arange(N) + 11, (N + 12,) + (3,) * (axes - 1)), 1).astype(np.float32)
    return rng.uniform(-1000, 1000, (N, axes)).astype(np.float32)


@pytest.mark.parametrize("layout", ["pairs", "halves", "sections"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,D,dims", [(1, 32, (32,)), (4, 32, (16, 16)), (8, 64, (16, 24, 24)), (2, 128, (32, 32, 32, 32)),
                                      (2, 64, (6, 10)), (3, 40, (4, 2, 10)), (1, 2, (2,)), (5, 6, (2, 2)), (2, 256, (128, 64)),
                                      (1, 512, (128, 128, 128, 128)), (2, 512, (510,)), (16, 80, (16, 32, 32)), (2, 96, (32, 64))])
def test_turns(H, D, dims, dtype, layout):
    N = 67
    Q, K, _ = synth.features(H * D, N, H, D, dtype)
    for inverse in (False, True):
        pos = positions(H + D, N, len(dims), "grid" if inverse else "points")
        q, k = run(pos, Q, dims, K, layout=layout, inverse=inverse)
        check(q, pos, Q, dims, 10000.0, layout, inverse, dtype)
        check(k, pos, K, dims, 10000.0, layout, inverse, dtype)
        q1, _ = run(pos, Q, dims, layout=layout, inverse=inverse)
        assert np.array_equal(q1, q)
        q2, k2 = run(pos, Q, dims, K, layout=layout, inverse=inverse, in_place=True)
        assert np.array_equal(q2, q) and np.array_equal(k2, k)


@pytest.mark.parametrize("N", [1, 2, 255, 256, 257, 5000])
def test_node_counts(N):
    Q, K, _ = synth.features(N, N, 2, 32, "bf16")
    pos = positions(N, N, 2, "points")
    q, k = run(pos, Q, (8, 24), K, theta=100.0, layout="halves")
    check(q, pos, Q, (8, 24), 100.0, "halves", False, "bf16")
    check(k, pos, K, (8, 24), 100.0, "halves", False, "bf16")


def test_far_positions():
    # up to the last whole numbers that fp32 holds, and far beyond them
    pos = np.array([[2.0 ** 24 - 1], [-2.0 ** 24 + 3], [123456.78], [1e9], [-3e11], [1e-30], [0.0]], np.float32)
    Q = synth.features(4, len(pos), 2, 32, "f32")[0]
    q, _ = run(pos, Q, (32,))
    # (the turns' own rounding in 64 bits: 2^-53 of the angle, in the oracle's angle too)
    want, size = ref.rope(pos, Q, (32,), 10000.0, "pairs", False)
    far = np.abs(pos.astype(np.float64))[:, :, None] * 2.0 ** -50
    assert np.all(np.abs(q - want) <= (TRIG + far) * size + ref.ROUND["f32"] * np.abs(want))
    assert np.array_equal(q[-1], Q[-1])  # position 0 turns nothing


def test_positions_that_are_not_finite():
    N, dims = 20, (8, 16)
    Q = synth.features(6, N, 2, 32, "f32")[0]
    pos = positions(6, N, 2, "points")
    pos[3, 0], pos[7, 1], pos[9] = np.nan, np.inf, -np.inf
    q, _ = run(pos, Q, dims)
    bad = np.zeros((N, 32), bool)
    bad[3, :8] = bad[7, 8:24] = bad[9, :24] = True
    assert np.array_equal(np.isnan(q), np.broadcast_to(bad[:, None], q.shape))
    assert np.array_equal(q[[3, 7, 9], :, 24:], Q[[3, 7, 9], :, 24:])


def test_inverse_is_the_gradient():
    # <turn(x), y> = <x, turn back(y)>
    N, dims = 500, (16, 24, 24)
    Q, Y, _ = synth.features(8, N, 4, 64, "f32")
    pos = positions(8, N, 3, "grid")
    a, b = run(pos, Q, dims)[0], run(pos, Y, dims, inverse=True)[0]
    lhs, rhs = np.sum(a.astype(np.float64) * Y, -1), np.sum(Q.astype(np.float64) * b, -1)
    assert np.max(np.abs(lhs - rhs)) <= 64 * 2 * 3 * 2 ** -20 * np.max(np.abs(Q)) * np.max(np.abs(Y))
