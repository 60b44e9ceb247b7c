"""Differential attention on the GPU, forward and backward, through the C ABI
against the float64 form of tests/layer_ref.py, with its tolerances."""
import math

import numpy as np
import pytest

import synth
from tests import layer_ref as ref
from tests.helpers import to_device, to_host_f32

pytestmark = pytest.mark.gpu

CASES = [(h, d, t) for h in (1, 2, 4, 8) for d in (32, 64, 128) for t in ("f32", "bf16")] + [(1, 256, "bf16"), (4, 256, "bf16")]
FORCED_SPLIT = {"light_max_deg": 2, "heavy_min_deg": 6, "chunk_edges": 64, "grid_blocks": 0}


def inputs(seed, N, H, D, dtype, graph=None, std=1.0):
    rowptr, colidx = graph or synth.ragged_graph(seed, N, max_deg=24, empty_frac=0.1,
                                                 hubs={h: d for h, d in {7: 299, 100: 150, 299: 70}.items() if h < N and d < N},
                                                 self_loops=False, dup_frac=0.05, shuffle=True)
    Q, K, V = synth.features(seed, N, 2 * H, D, dtype)
    dO = synth.features(seed + 1, N, H, 2 * D, dtype)[0]
    if dtype == "f32":
        Q = Q * np.float32(std)
    lam = (np.linspace(-0.4, 0.9, H) if H > 1 else np.array([0.7])).astype(np.float32)
    return rowptr, colidx, Q, K, V.reshape(N, H, 2 * D), lam, dO, np.float32(1 / math.sqrt(D))


def larger_graph(seed, H, D, dtype):
    """Enough rows and entries that the call partitions its rows: short rows, hubs, empty rows."""
    row = 2 * H * D * (4 if dtype == "f32" else 2)
    entries = min(32768, (16 << 20) // row) + 1000
    N = max(600, entries // 12)
    return synth.ragged_graph(seed, N, max_deg=24, empty_frac=0.1, hubs={7: 599, 100: 150, 299: 70}, self_loops=True, dup_frac=0.05,
                              shuffle=True)


def run_fwd(rowptr, colidx, Q, K, V, lam, scale, tuning=None, want_lse=True):
    import torch
    import paper_2605_31500_amd as gt
    rp, ci, q, k, v, lm = (to_device(x) for x in (rowptr, colidx, Q, K, V, lam))
    out = torch.full_like(v, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), device=q.device) if want_lse else None
    gt.gt_diff_attn_fwd(rp, ci, q, k, v, lm, out, scale, tuning=tuning, lse=lse)
    torch.cuda.synchronize()
    return to_host_f32(out), lse.cpu().numpy() if want_lse else None


def run_bwd(rowptr, colidx, Q, K, V, lam, dO, lse, scale, want_dlam=True):
    import torch
    import paper_2605_31500_amd as gt
    rpt, cit = synth.transpose_csr(rowptr, colidx, Q.shape[0])
    rp, ci, rt, ct, q, k, v, lm, do, ls = (to_device(x) for x in (rowptr, colidx, rpt, cit, Q, K, V, lam, dO, lse))
    dq, dk, dv = (torch.full_like(x, float("nan")) for x in (q, k, v))
    dl = torch.full_like(lm, float("nan")) if want_dlam else None
    gt.gt_diff_attn_bwd(rp, ci, rt, ct, q, k, v, lm, do, ls, dq, dk, dv, dl, scale)
    torch.cuda.synchronize()
    return to_host_f32(dq), to_host_f32(dk), to_host_f32(dv), dl.cpu().numpy() if want_dlam else None


def check_fwd(x, dtype, tuning=None):
    rowptr, colidx, Q, K, V, lam, _, scale = x
    out, lse = run_fwd(rowptr, colidx, Q, K, V, lam, scale, tuning)
    r = ref.Diff(rowptr, colidx, Q, K, V, lam, scale)
    b = ref.DiffBounds(rowptr, colidx, Q, K, scale, dtype, r.lse)
    assert ref.worst(out, r.out, r.Sout, b.out) <= 1
    fin = np.isfinite(r.lse)
    assert np.array_equal(np.isneginf(lse), ~fin)
    assert np.all(np.abs(lse[fin] - r.lse[fin]) <= b.lse[fin])
    return out, lse


def check_bwd(x, dtype):
    rowptr, colidx, Q, K, V, lam, dO, scale = x
    lse = ref.Diff(rowptr, colidx, Q, K, V, lam, scale).lse.astype(np.float32)
    r = ref.Diff(rowptr, colidx, Q, K, V, lam, scale, dO, lse)
    b = ref.DiffBounds(rowptr, colidx, Q, K, scale, dtype, lse)
    got = run_bwd(rowptr, colidx, Q, K, V, lam, dO, lse, scale)
    for name, g in zip(("dQ", "dK", "dV", "dlam"), got):
        err = ref.worst(g, getattr(r, name), getattr(r, "S" + name), getattr(b, name))
        assert err <= 1, "%s: %.3g of its tolerance" % (name, err)
    return got


@pytest.mark.parametrize("split", [False, True], ids=["default", "forced_split"])
@pytest.mark.parametrize("H,D,dtype", CASES)
def test_forward(H, D, dtype, split):
    check_fwd(inputs(100 * H + D, 300, H, D, dtype), dtype, FORCED_SPLIT if split else None)


@pytest.mark.parametrize("H,D,dtype", CASES)
def test_backward(H, D, dtype):
    check_bwd(inputs(200 * H + D, 300, H, D, dtype), dtype)


@pytest.mark.parametrize("H,D,dtype", CASES)
def test_larger_graph(H, D, dtype):
    g = larger_graph(H + D, H, D, dtype)
    x = inputs(300 * H + D, g[0].size - 1, H, D, dtype, g)
    check_fwd(x, dtype)
    check_bwd(x, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 63, 65])
def test_few_rows(N, dtype):
    x = inputs(300 + N, N, 2, 32, dtype, synth.ragged_graph(300 + N, N, max_deg=3, empty_frac=0.3, self_loops=N == 1))
    check_fwd(x, dtype)
    check_bwd(x, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph_without_entries(dtype):
    N, H, D = 70, 2, 32
    x = inputs(9, N, H, D, dtype, (np.zeros(N + 1, np.int64), np.zeros(0, np.int32)))
    out, lse = run_fwd(*x[:6], x[7])
    assert np.all(out == 0) and np.all(np.isneginf(lse))
    for g in run_bwd(*x[:6], x[6], lse, x[7]):
        assert np.all(g == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("deg", [150, 1500])
def test_long_rows(deg, dtype):
    # every row long: cut into pieces on all XCDs (deg 1500: spread over a wave's groups too)
    N = 2000 if deg == 150 else 1600
    g = synth.csr_from_degrees(11, N, np.full(N, deg), self_loops=False) if deg == 150 else synth.ragged_graph(
        12, N, max_deg=4, hubs={i: 1500 for i in range(0, 40)}, shuffle=True)
    x = inputs(13, N, 1, 64, dtype, g)
    check_fwd(x, dtype)
    check_bwd(x, dtype)


@pytest.mark.parametrize("split", [False, True], ids=["default", "forced_split"])
def test_peaked_scores(split):
    # scores of hundreds: most weights underflow, one or two entries carry a row
    x = inputs(14, 300, 2, 32, "f32", std=80.0)
    check_fwd(x, "f32", FORCED_SPLIT if split else None)
    check_bwd(x, "f32")


def test_first_entry_of_no_weight_and_large_value():
    # the mean that the backward takes off starts at a value that does not count
    N, deg = 300, 9
    rowptr = np.arange(N + 1, dtype=np.int64) * deg
    colidx = (1 + (np.arange(N)[:, None] * 7 + np.arange(deg) * 31) % (N - 1)).astype(np.int32)
    colidx[:, 0] = 0
    x = inputs(15, N, 1, 32, "f32", (rowptr, colidx.reshape(-1)))
    Q, K, V = x[2:5]
    Q[..., 0], K[0], V[0] = 3, 0, 1e4
    K[0, :, 0] = -40  # a score of -21: a weight of about 1e-10
    check_bwd(x, "f32")


def test_one_entry_per_row():
    # out = (1 - lambda) V of the entry, no gradient of queries and keys
    N, H, D = 500, 2, 32
    x = inputs(16, N, H, D, "f32", synth.csr_from_degrees(16, N, np.ones(N, np.int64), self_loops=False))
    out, _ = check_fwd(x, "f32")
    lam = x[5].astype(np.float64)[None, :, None]
    assert np.all(np.abs(out - ((1 - lam) * x[4][x[1]])) <= 2.0 ** -23 * np.abs(x[4][x[1]]))
    dq, dk, _, _ = check_bwd(x, "f32")
    assert np.all(dq == 0)
    assert np.max(np.abs(dk)) <= 1e-4


@pytest.mark.parametrize("split", [False, True], ids=["default", "forced_split"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_minus_infinity(dtype, split):
    """Sources that every query scores -inf have weight 0, wherever they stand in
    a row, and a row of such sources alone counts as empty in that map."""
    N, H, D = 300, 2, 32
    rowptr, colidx, Q, K, V, lam, dO, scale = inputs(17, N, H, D, dtype)
    one = np.float32(1.0) if dtype == "f32" else np.uint16(0x3F80)
    ninf = np.float32(-np.inf) if dtype == "f32" else np.uint16(0xFF80)
    Q[..., 0] = one  # the masked sources' first element decides: 1 * -inf
    masked = np.zeros(N, bool)
    masked[::2] = True
    masked[colidx[rowptr[20]:rowptr[30]]] = True  # rows 20..29: nothing left
    K[masked, 0::2, 0] = ninf  # the first map alone
    K[masked, 0::2, 1:] = 0
    out, lse = run_fwd(rowptr, colidx, Q, K, V, lam, scale, FORCED_SPLIT if split else None)
    r = ref.Diff(rowptr, colidx, Q, K, V, lam, scale)
    kz = K.copy()
    kz[masked, 0::2, 0] = 0
    b = ref.DiffBounds(rowptr, colidx, Q, kz, scale, dtype, r.lse)
    assert np.array_equal(np.isneginf(lse), np.isneginf(r.lse)) and np.isneginf(lse[25, 0])
    assert ref.worst(out, r.out, r.Sout, b.out) <= 1
    # gradients: of no weight, but 0 * -inf where a key itself is not finite
    got = run_bwd(rowptr, colidx, Q, K, V, lam, dO, r.lse.astype(np.float32), scale)
    with np.errstate(invalid="ignore"):
        r = ref.Diff(rowptr, colidx, Q, K, V, lam, scale, dO, r.lse.astype(np.float32))
    assert ref.worst(got[2], r.dV, r.SdV, b.dV) <= 1
    assert ref.worst(got[3], r.dlam, r.Sdlam, b.dlam) <= 1
    assert ref.worst(got[1], r.dK, r.SdK, b.dK) <= 1
    assert ref.worst(got[0][:, 1::2], r.dQ[:, 1::2], r.SdQ[:, 1::2], np.broadcast_to(b.dQ, r.dQ.shape)[:, 1::2]) <= 1
    fin = np.isfinite(r.dQ) & np.isfinite(r.SdQ)
    x, y, s = (np.where(fin, z, 0.0) for z in (got[0], r.dQ, r.SdQ))
    assert ref.worst(x, y, s, b.dQ) <= 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_non_finite_sources_stay_with_their_rows(dtype):
    N, H, D = 300, 2, 32
    rowptr, colidx, Q, K, V, lam, _, scale = inputs(18, N, H, D, dtype)
    clean, _ = run_fwd(rowptr, colidx, Q, K, V, lam, scale)
    nan = np.float32(np.nan) if dtype == "f32" else np.uint16(0x7FC0)
    bad = np.array([5, 77, 123])
    K[bad[0], 1, 3] = nan
    V[bad[1:], 0, 5] = nan
    out, _ = run_fwd(rowptr, colidx, Q, K, V, lam, scale)
    names = np.zeros((N, 3), bool)
    for b in range(3):
        np.logical_or.at(names[:, b], ref.rows_of(rowptr), colidx == bad[b])
    assert np.all(np.isnan(out[names[:, 0], 0]))
    assert np.all(np.isnan(out[names[:, 1] | names[:, 2], 0, 5]))
    keep = ~names.any(1)
    assert np.array_equal(out[keep], clean[keep]) and np.array_equal(out[~names[:, 0], 1], clean[~names[:, 0], 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lambda_zero_is_the_softmax_attention(dtype):
    """lambda = 0: the first map alone, as gt_attn_fwd computes it for the first half of the values."""
    import paper_2605_31500_amd as gt
    N, H, D = 300, 2, 32
    rowptr, colidx, Q, K, V, lam, _, scale = inputs(19, N, H, D, dtype)
    out, lse = run_fwd(rowptr, colidx, Q, K, V, np.zeros_like(lam), scale)
    q, k, v = (np.ascontiguousarray(x) for x in (Q[:, 0::2], K[:, 0::2], V[..., :D]))
    rp, ci, q, k, v = (to_device(x) for x in (rowptr, colidx, q, k, v))
    want, wl = gt.attention(rp, ci, q, k, v, scale, return_lse=True)
    tol = ref.DiffBounds(rowptr, colidx, Q, K, scale, dtype, lse).out
    r = ref.Diff(rowptr, colidx, Q, K, V, np.zeros_like(lam), scale)
    assert np.all(np.abs(out[..., :D] - to_host_f32(want)) <= 2 * tol * np.maximum(r.Sout[..., :D], 1e-30))
    fin = np.isfinite(lse[:, 0::2])
    assert np.allclose(lse[:, 0::2][fin], wl.cpu().numpy()[fin], rtol=1e-5, atol=1e-5)


def test_deterministic_and_optional_outputs():
    x = inputs(20, 300, 2, 64, "bf16")
    a, la = run_fwd(*x[:6], x[7])
    b, _ = run_fwd(*x[:6], x[7], want_lse=False)
    assert np.array_equal(a, b)
    g1, g2 = run_bwd(*x[:6], x[6], la, x[7]), run_bwd(*x[:6], x[6], la, x[7], want_dlam=False)
    for p, q in zip(g1[:3], g2[:3]):
        assert np.array_equal(p, q)
    assert np.array_equal(g1[3], run_bwd(*x[:6], x[6], la, x[7])[3])


def test_entries_repeated_many_times():
    # one source over and over: atomics-free sums, weights 1/d each
    N, d = 40, 700
    rowptr = np.arange(N + 1, dtype=np.int64) * d
    colidx = np.repeat(np.arange(N, dtype=np.int32)[::-1], d).copy()
    x = inputs(21, N, 1, 32, "f32", (rowptr, colidx))
    check_fwd(x, "f32")
    check_bwd(x, "f32")
