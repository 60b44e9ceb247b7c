"""Layer norm on the GPU, forward and backward, through the C ABI against the
float64 form of tests/layer_ref.py, with its tolerances."""
import numpy as np
import pytest

import synth
from tests import layer_ref as ref
from tests.helpers import to_device, to_host_f32

pytestmark = pytest.mark.gpu

EPS = 1e-5
WIDTHS = [1, 2, 3, 7, 8, 31, 64, 65, 96, 127, 128, 200, 203, 256, 384, 500, 512, 768, 1000, 1023, 1024, 1280, 2048, 2056, 4096, 4099,
          5000, 8192, 10001, 16384]


def inputs(seed, N, F, dtype, offset=0.5):
    X = synth.normal(seed, 1, (N, F), 1.0, "f32") + np.float32(offset) * synth.normal(seed, 2, (1, F), 1.0, "f32")
    X = (X * np.exp(0.4 * synth.normal(seed, 3, (N, 1), 1.0, "f32"))).astype(np.float32)
    dO = synth.normal(seed, 4, (N, F), 1.0, "f32")
    gamma = (1 + 0.3 * synth.normal(seed, 5, (F,), 1.0, "f32")).astype(np.float32)
    beta = (0.3 * synth.normal(seed, 6, (F,), 1.0, "f32")).astype(np.float32)
    if dtype == "bf16":
        X, dO = (((x.view(np.uint32) + 0x8000) >> 16).astype(np.uint16) for x in (X, dO))
    return X, dO, gamma, beta


def dev(x):
    return None if x is None else to_device(x)


def run_fwd(X, gamma, beta, eps=EPS, stats=True, in_place=False):
    import torch
    import paper_2605_31500_amd as gt
    x, g, b = dev(X), dev(gamma), dev(beta)
    out = x if in_place else torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((X.shape[0],), float("nan"), device=x.device) for _ in range(2)) if stats else (None, None)
    gt.gt_layernorm_fwd(x, g, b, out, eps, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    return to_host_f32(out), *((mean.cpu().numpy(), rstd.cpu().numpy()) if stats else (None, None))


def run_bwd(X, dO, gamma, mean, rstd, params=(True, True), into=None):
    import torch
    import paper_2605_31500_amd as gt
    x, do, g, m, r = dev(X), dev(dO), dev(gamma), dev(mean), dev(rstd)
    dx = {"X": x, "dout": do}.get(into)
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    dg, db = (torch.full((X.shape[1],), float("nan"), device=x.device) if p else None for p in params)
    gt.gt_layernorm_bwd(x, do, g, m, r, dx, dgamma=dg, dbeta=db)
    torch.cuda.synchronize()
    return to_host_f32(dx), None if dg is None else dg.cpu().numpy(), None if db is None else db.cpu().numpy()


def check(X, dO, gamma, beta, dtype, eps=EPS):
    N = X.shape[0]
    r = ref.Norm(X, gamma, beta, eps)
    out, mean, rstd = run_fwd(X, gamma, beta, eps)
    assert ref.worst(mean, r.mean, r.Smean, r.sums) <= 1
    assert ref.worst(rstd, r.rstd, r.Srstd, r.sums) <= 1
    assert ref.worst(out, r.out, r.Sout, r.sums + ref.ROUND[dtype]) <= 1
    m, s = r.mean.astype(np.float32), r.rstd.astype(np.float32)
    r = ref.Norm(X, gamma, beta, eps, dO, m, s)
    dx, dg, db = run_bwd(X, dO, gamma, m, s)
    assert ref.worst(dx, r.dX, r.SdX, r.sums + ref.ROUND[dtype]) <= 1
    assert ref.worst(dg, r.dgamma, r.Sdgamma, (N + 16) * ref.U32) <= 1
    assert ref.worst(db, r.dbeta, r.Sdbeta, (N + 16) * ref.U32) <= 1
    return out, mean, rstd, dx, dg, db


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", WIDTHS)
def test_widths(F, dtype):
    check(*inputs(F, 37, F, dtype), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [32, 100, 128, 203, 1024])
@pytest.mark.parametrize("N", [1, 2, 255, 1025, 2999])
def test_row_counts(N, F, dtype):
    check(*inputs(N + F, N, F, dtype), dtype)


@pytest.mark.parametrize("F", [64, 203, 512])
def test_optional_parameters_and_outputs(F):
    X, dO, gamma, beta = inputs(F, 300, F, "f32")
    for g, b in ((None, None), (gamma, None), (None, beta)):
        r = ref.Norm(X, g, b, EPS)
        out, mean, rstd = run_fwd(X, g, b)
        assert ref.worst(out, r.out, r.Sout, r.sums + ref.U32) <= 1
        assert np.array_equal(run_fwd(X, g, b, stats=False)[0], out)
    r = ref.Norm(X, None, None, EPS, dO, mean, rstd)
    full = run_bwd(X, dO, None, mean, rstd)
    assert ref.worst(full[0], r.dX, r.SdX, r.sums + ref.U32) <= 1
    for params in ((True, False), (False, True), (False, False)):
        part = run_bwd(X, dO, None, mean, rstd, params)
        assert np.array_equal(part[0], full[0])
        for k in range(2):
            assert part[k + 1] is None or np.array_equal(part[k + 1], full[k + 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [100, 203, 256, 2048, 6000])
def test_in_place(F, dtype):
    X, dO, gamma, beta = inputs(F, 200, F, dtype)
    out, mean, rstd = run_fwd(X, gamma, beta)
    assert np.array_equal(run_fwd(X, gamma, beta, in_place=True)[0], out)
    want = run_bwd(X, dO, gamma, mean, rstd)
    for into in ("X", "dout"):
        for a, b in zip(run_bwd(X, dO, gamma, mean, rstd, into=into), want):
            assert np.array_equal(a, b)


def test_constant_rows_and_large_offsets():
    X, dO, gamma, beta = inputs(1, 64, 256, "f32")
    X[:8] = np.arange(8, dtype=np.float32)[:, None] * 3  # variance 0
    X[8:16] += np.float32(4096)  # a mean far above the spread
    check(X, dO, gamma, beta, "f32", eps=1e-3)
    out = run_fwd(X, gamma, beta, 1e-3)[0]
    assert np.max(np.abs(out[:8] - beta)) <= 1e-3


def test_rows_that_are_not_finite_stay_alone():
    X, dO, gamma, beta = inputs(2, 300, 203, "f32")
    clean = run_fwd(X, gamma, beta)[0]
    X[5, 7], X[100, 0], X[299, 202] = np.nan, np.inf, -np.inf
    out = run_fwd(X, gamma, beta)[0]
    bad = [5, 100, 299]
    assert np.all(np.isnan(out[bad]).any(1))
    keep = np.setdiff1d(np.arange(300), bad)
    assert np.array_equal(out[keep], clean[keep])


@pytest.mark.parametrize("N,F,dtype", [(300000, 8, "bf16"), (70001, 33, "f32"), (20000, 512, "f32")])
def test_many_rows(N, F, dtype):
    # (the parameters' gradients: sums of at most N / 256 + 256 terms in fp32)
    X, dO, gamma, beta = inputs(N, N, F, dtype)
    r0 = ref.Norm(X, gamma, beta, EPS)
    m, s = r0.mean.astype(np.float32), r0.rstd.astype(np.float32)
    r = ref.Norm(X, gamma, beta, EPS, dO, m, s)
    out = run_fwd(X, gamma, beta)[0]
    assert ref.worst(out, r0.out, r0.Sout, r0.sums + ref.ROUND[dtype]) <= 1
    dx, dg, db = run_bwd(X, dO, gamma, m, s)
    again = run_bwd(X, dO, gamma, m, s)
    assert ref.worst(dx, r.dX, r.SdX, r.sums + ref.ROUND[dtype]) <= 1
    assert ref.worst(dg, r.dgamma, r.Sdgamma, (N / 256 + 272) * ref.U32) <= 1
    assert ref.worst(db, r.dbeta, r.Sdbeta, (N / 256 + 272) * ref.U32) <= 1
    assert all(np.array_equal(a, b) for a, b in zip((dx, dg, db), again))


def test_no_rows_set_the_parameters_gradients():
    import torch
    import paper_2605_31500_amd as gt
    x, s = torch.empty((0, 40), device="cuda"), torch.empty(0, device="cuda")
    dg, db = torch.full((40,), 3.0, device="cuda"), torch.full((40,), 3.0, device="cuda")
    gt.gt_layernorm_fwd(x, None, None, x, EPS)
    gt.gt_layernorm_bwd(x, x, None, s, s, x, dgamma=dg, dbeta=db)
    lam, dlam = torch.ones(2, device="cuda"), torch.full((2,), 3.0, device="cuda")
    q, v = torch.empty((0, 4, 32), device="cuda"), torch.empty((0, 2, 64), device="cuda")
    rp, ci = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    gt.gt_diff_attn_bwd(rp, ci, rp, ci, q, q, v, lam, v, torch.empty((0, 4), device="cuda"), q, q, v, dlam, 1.0)
    gt.gt_rope(torch.empty((0, 1), device="cuda"), q, q, [32])
    torch.cuda.synchronize()
    assert torch.all(dg == 0) and torch.all(db == 0) and torch.all(dlam == 0)
