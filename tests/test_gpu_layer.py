"""The operators of include/gt_layer.h used together and as programs use them:
a differential attention block forward and backward against the composition of
the plain float64 forms, its gradients against differences, calls captured into
HIP graphs and replayed, on streams of their own, from several host threads, and
rows past a call's tensors left as they were."""
import math
import threading

import numpy as np
import pytest

import synth
from tests import layer_ref as ref
from tests.helpers import to_device, to_host_f32

pytestmark = pytest.mark.gpu

DIMS = (8, 12, 12)


def block_inputs(seed, N, dtype):
    H, D = 2, 32
    rowptr, colidx = synth.ragged_graph(seed, N, max_deg=12, empty_frac=0.1, hubs={5: min(N - 1, 200)} if N > 5 else None,
                                        self_loops=N < 5, shuffle=True)
    Q, K, V = synth.features(seed, N, 2 * H, D, dtype)
    rng = np.random.default_rng(seed)
    return dict(rowptr=rowptr, colidx=colidx, Q=Q, K=K, V=V.reshape(N, H, 2 * D), lam=np.array([0.3, 0.8], np.float32),
                pos=rng.integers(0, 30, (N, 3)).astype(np.float32), gamma=(1 + 0.2 * rng.standard_normal(2 * D)).astype(np.float32),
                beta=(0.2 * rng.standard_normal(2 * D)).astype(np.float32), dO=synth.features(seed + 1, N, H, 2 * D, dtype)[0])


def run_block(x, stream=None):
    """The block's convenience functions; `stream`: on a stream that is not the current one."""
    import torch
    import paper_2605_31500_amd as gt
    N = x["Q"].shape[0]
    d = {k: to_device(v) for k, v in x.items()}
    rt, ct = (to_device(t) for t in synth.transpose_csr(x["rowptr"], x["colidx"], N))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    out, saved = gt.diff_attention(d["rowptr"], d["colidx"], d["Q"], d["K"], d["V"], d["lam"], pos=d["pos"], dims=DIMS, theta=100.0,
                                   layout="halves", norm=(d["gamma"], d["beta"]), return_saved=True, stream=stream)
    grads = gt.diff_attention_bwd(d["rowptr"], d["colidx"], rt, ct, saved, d["dO"], stream=stream)
    torch.cuda.synchronize()
    return to_host_f32(out), {k: to_host_f32(v) for k, v in grads.items()}


def plain_block(x, dO=None):
    """The block in float64: output, and gradients for dO."""
    N, maps, D = x["Q"].shape
    H = maps // 2
    scale = np.float32(D ** -0.5)
    q, k = (ref.rope(x["pos"], x[n], DIMS, 100.0, "halves", False)[0] for n in ("Q", "K"))
    v, lam = ref.widen(x["V"]), x["lam"]
    att = ref.Diff(x["rowptr"], x["colidx"], q, k, v, lam, scale)
    rows = att.out.reshape(N * H, -1)
    norm = ref.Norm(rows, x["gamma"], x["beta"], 1e-5)
    out = norm.out.reshape(N, H, -1)
    if dO is None:
        return out
    nb = ref.Norm(rows, x["gamma"], x["beta"], 1e-5, ref.widen(dO).reshape(N * H, -1), norm.mean, norm.rstd)
    ab = ref.Diff(x["rowptr"], x["colidx"], q, k, v, lam, scale, nb.dX.reshape(N, H, -1))
    dq, dk = (ref.rope(x["pos"], g, DIMS, 100.0, "halves", True)[0] for g in (ab.dQ, ab.dK))
    return out, dict(dQ=dq, dK=dk, dV=ab.dV, dlam=ab.dlam, dgamma=nb.dgamma, dbeta=nb.dbeta), ab.Sdlam


def near(a, b, tol):
    return float(np.linalg.norm(a.astype(np.float64) - b)) <= tol * float(np.linalg.norm(b)) + 1e-9


# Norm of the difference: the chain rounds its values at most eight times on the
# way to a gradient (turned queries, output, normalised rows, their gradient, the
# turned back ones ...), which the softmax and the norm amplify by no more than
# four here (scores of order 1, unit gains): 8 * 4 half steps of the type.
# (Rows of one entry are near a constant multiple of a value row, whose norm is of order 1.)
TOL = {"f32": 32 * 2.0 ** -24 * 8, "bf16": 32 * 2.0 ** -8}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 40, 500, 5000])
def test_block_forward_and_backward(N, dtype):
    x = block_inputs(N, N, dtype)
    out, grads = run_block(x)
    want, wgrads, Sdlam = plain_block(x, x["dO"])
    assert near(out, want, TOL[dtype])
    assert set(grads) == set(wgrads)
    for k, g in grads.items():
        assert np.all(np.isfinite(g)) and g.shape == wgrads[k].shape
        if k != "dlam":
            assert near(g, wgrads[k], TOL[dtype]), k
    # dlam is minus the sum of sum_e a_1,e <dout_i, V_j> over rows, each product of which is off by TOL of itself:
    # so dlam is off by TOL of the sum of their absolute values, Sdlam.  Of its own value it may be off by any
    # factor: a row of one entry is (1 - lambda) V, which the norm makes independent of lambda but for eps, so its
    # products add up to nearly 0 (one row, fp32: |dlam| 7e-4 and 0.025 of Sdlam 70 and 156, where TOL Sdlam is 1.1e-3 and 2.4e-3).
    assert np.all(np.abs(grads["dlam"] - wgrads["dlam"]) <= TOL[dtype] * Sdlam)


def test_block_gradients_against_differences():
    x = block_inputs(3, 60, "f32")
    _, grads = run_block(x)
    rng = np.random.default_rng(1)
    for name, key in (("Q", "dQ"), ("K", "dK"), ("V", "dV"), ("lam", "dlam"), ("gamma", "dgamma"), ("beta", "dbeta")):
        step = rng.standard_normal(x[name].shape)
        vals = []
        for sign in (1, -1):
            y = dict(x)
            y[name] = x[name].astype(np.float64) + sign * 1e-6 * step
            vals.append(float(np.sum(plain_block(y) * x["dO"])))
        want = (vals[0] - vals[1]) / 2e-6
        # (the differences' own error is of order 1e-9 over the step; the kernels' fp32 one of the sum's terms)
        assert abs(float(np.sum(grads[key] * step)) - want) <= 1e-4 * float(np.sum(np.abs(grads[key] * step))) + 1e-3, name


def test_block_on_another_stream():
    import torch
    x = block_inputs(6, 5000, "f32")
    want, wgrads = run_block(x)
    for _ in range(3):
        out, grads = run_block(x, torch.cuda.Stream())
        assert np.array_equal(out, want) and all(np.array_equal(grads[k], wgrads[k]) for k in wgrads)


def test_block_without_rows():
    import torch
    import paper_2605_31500_amd as gt
    q, v, lam = torch.empty((0, 4, 32), device="cuda"), torch.empty((0, 2, 64), device="cuda"), torch.ones(2, device="cuda")
    rp, ci = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    out, saved = gt.diff_attention(rp, ci, q, q, v, lam, pos=torch.empty((0, 1), device="cuda"), norm=(None, None), return_saved=True)
    grads = gt.diff_attention_bwd(rp, ci, rp, ci, saved, out)
    torch.cuda.synchronize()
    assert out.shape == v.shape and torch.all(grads["dlam"] == 0)


def test_attention_turns_queries_and_keys():
    import paper_2605_31500_amd as gt
    x = block_inputs(4, 300, "f32")
    d = {k: to_device(v) for k, v in x.items()}
    got = gt.attention(d["rowptr"], d["colidx"], d["Q"], d["K"], d["V"].view(d["Q"].shape), pos=d["pos"], dims=DIMS, layout="sections")
    q, k = (ref.rope(x["pos"], x[n], DIMS, 10000.0, "sections", False)[0].astype(np.float32) for n in ("Q", "K"))
    want = gt.attention(d["rowptr"], d["colidx"], to_device(q), to_device(k), d["V"].view(d["Q"].shape))
    # scores of both differ by at most 64 elements' 2^-21 turns: 1e-4 of values of order 1
    assert np.max(np.abs(to_host_f32(got) - to_host_f32(want))) <= 1e-3


def calls_of(x, d, outs):
    """One call of each operator on device inputs d, into outs."""
    import paper_2605_31500_amd as gt
    s = float(np.float32(x["Q"].shape[-1] ** -0.5))
    f = d["X"]
    gt.gt_rope(d["pos"], d["Q"], outs["rq"], DIMS, K=d["K"], out_k=outs["rk"], layout="halves")
    gt.gt_diff_attn_fwd(d["rowptr"], d["colidx"], outs["rq"], outs["rk"], d["V"], d["lam"], outs["out"], s, lse=outs["lse"])
    gt.gt_layernorm_fwd(f, None, None, outs["y"], mean=outs["mean"], rstd=outs["rstd"])
    gt.gt_layernorm_bwd(f, d["dX"], None, outs["mean"], outs["rstd"], outs["dx"], dgamma=outs["dgamma"], dbeta=outs["dbeta"])
    gt.gt_diff_attn_bwd(d["rowptr"], d["colidx"], d["rt"], d["ct"], outs["rq"], outs["rk"], d["V"], d["lam"], d["dO"], outs["lse"],
                        outs["dq"], outs["dk"], outs["dv"], outs["dlam"], s)


def device_inputs(x):
    import torch
    d = {k: to_device(v) for k, v in x.items()}
    d["rt"], d["ct"] = (to_device(t) for t in synth.transpose_csr(x["rowptr"], x["colidx"], x["Q"].shape[0]))
    N = x["Q"].shape[0]
    d["X"], d["dX"] = (to_device(synth.normal(N, 7 + i, (N, 203), 1.0, "bf16")) for i in range(2))
    outs = dict(rq=d["Q"], rk=d["K"], out=d["V"], y=d["X"], dx=d["X"], dq=d["Q"], dk=d["K"], dv=d["V"], dlam=d["lam"])
    outs = {k: torch.empty_like(v) for k, v in outs.items()}
    for k, shape in (("lse", d["Q"].shape[:2]), ("mean", (N,)), ("rstd", (N,)), ("dgamma", (203,)), ("dbeta", (203,))):
        outs[k] = torch.empty(shape, device="cuda")
    return d, outs


@pytest.mark.parametrize("N", [300, 6000])
def test_captured_and_replayed(N):
    """Two graphs of the same calls, replayed in turn with eager work between:
    every replay equals the eager results bit for bit."""
    import torch
    x = block_inputs(N, N, "f32")
    d, want = device_inputs(x)
    calls_of(x, d, want)
    torch.cuda.synchronize()
    runs = []
    for _ in range(2):
        _, outs = device_inputs(x)
        g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=s):
            calls_of(x, d, outs)
        runs.append((g, outs))
    _, eager = device_inputs(x)
    for _ in range(3):
        for g, outs in runs:
            for t in outs.values():
                t.fill_(float("nan"))
            g.replay()
            calls_of(x, d, eager)
            torch.cuda.synchronize()
            for k in want:
                assert torch.equal(outs[k], want[k]), k
                assert torch.equal(eager[k], want[k]), k


def test_streams_and_threads():
    """Four host threads, each on its own stream with its own graph, and two
    streams of one thread: as the same calls one after another."""
    import torch
    cases = []
    for i, N in enumerate((200, 3000, 6000, 9000)):
        x = block_inputs(50 + i, N, "bf16" if i % 2 else "f32")
        d, want = device_inputs(x)
        calls_of(x, d, want)
        cases.append((x, d, want, device_inputs(x)[1]))
    torch.cuda.synchronize()
    errors = []

    def work(x, d, outs):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(5):
                    calls_of(x, d, outs)
            s.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(x, d, outs)) for x, d, _, outs in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors and not any(t.is_alive() for t in threads)
    torch.cuda.synchronize()
    for _, _, want, outs in cases:
        for k in want:
            assert torch.equal(outs[k], want[k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,F", [(7, 203), (33, 100), (64, 129), (5, 1001), (9, 3)])
def test_rows_past_the_last_are_left(N, F, dtype):
    """Tensors that are the first rows of larger ones: what follows stays as it was."""
    import torch
    import paper_2605_31500_amd as gt
    x = to_device(synth.normal(N, 1, (N + 8, F), 1.0, dtype))
    dy = to_device(synth.normal(N, 2, (N + 8, F), 1.0, dtype))
    out, dx = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    mean, rstd = torch.full((N + 8,), 7.0, device="cuda"), torch.full((N + 8,), 7.0, device="cuda")
    dg, db = torch.full((F + 8,), 7.0, device="cuda"), torch.full((F + 8,), 7.0, device="cuda")
    gt.gt_layernorm_fwd(x[:N], None, None, out[:N], mean=mean[:N], rstd=rstd[:N])
    gt.gt_layernorm_bwd(x[:N], dy[:N], None, mean[:N], rstd[:N], dx[:N], dgamma=dg[:F], dbeta=db[:F])
    q = to_device(synth.features(N, N + 8, 3, 40, dtype)[0])
    oq = torch.full_like(q, 7.0)
    gt.gt_rope(torch.ones((N, 2), device="cuda"), q[:N], oq[:N], (6, 10), layout="halves")
    torch.cuda.synchronize()
    for t in (out[N:], dx[N:], mean[N:], rstd[N:], dg[F:], db[F:], oq[N:]):
        assert torch.all(t == 7.0)
    assert not torch.any(out[:N] == 7.0) and not torch.any(oq[:N] == 7.0)


def test_bench_modes():
    import json
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for op in ("diff", "diff-backward", "rope", "layernorm", "layernorm-backward"):
        r = subprocess.run([sys.executable, os.path.join(root, "bench.py"), "--config", "1", "--layer", op, "--steps", "3", "--warmup", "1"],
                           capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        line = json.loads(r.stdout.strip().splitlines()[-1])
        assert line["value"] > 0 and line["config"]["layer"] == op and line["roofline"]["frac"] > 0


# ------------------------------------------------------- offsets past 32 bits


def rows_of_bits(n, width, seed):
    """bf16 rows [n, width] made on the device, of more than 2^32 bytes."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty((n, width), dtype=torch.bfloat16, device="cuda")
    step = 1 << 17
    for a in range(0, n, step):
        x[a:a + step] = torch.randn((min(step, n - a), width), generator=g, device="cuda")
    return x


TAIL = 2048  # last rows, compared with a call on them alone


def test_layernorm_past_32_bits():
    import torch
    import paper_2605_31500_amd as gt
    n, f = 1_100_001, 2048  # 4.5 GB a tensor
    x, dy = rows_of_bits(n, f, 1), rows_of_bits(n, f, 2)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    out = torch.empty_like(x)
    gt.gt_layernorm_fwd(x, None, None, out, mean=mean, rstd=rstd)
    t = slice(n - TAIL, n)
    want, m, r = torch.empty_like(x[t]), torch.empty(TAIL, device="cuda"), torch.empty(TAIL, device="cuda")
    gt.gt_layernorm_fwd(x[t], None, None, want, mean=m, rstd=r)
    assert torch.equal(out[t], want) and torch.equal(mean[t], m) and torch.equal(rstd[t], r)
    dg, db = torch.empty(f, device="cuda"), torch.empty(f, device="cuda")
    gt.gt_layernorm_bwd(x, dy, None, mean, rstd, out, dgamma=dg, dbeta=db)
    gt.gt_layernorm_bwd(x[t], dy[t], None, m, r, want)
    assert torch.equal(out[t], want)
    ref = torch.zeros(f, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(ref)
    for a in range(0, n, 1 << 17):
        ref += dy[a:a + (1 << 17)].double().sum(0)
        size += dy[a:a + (1 << 17)].double().abs().sum(0)
    # (a lane sums at most n / 256 rows in fp32, workgroups' sums are added in 64 bits)
    assert bool(torch.all((db.double() - ref).abs() <= (n / 256 + 272) * 2.0 ** -24 * size))


@pytest.mark.parametrize("dims,layout", [((64, 96, 96), "halves"), ((62, 90, 90), "halves")])
def test_rope_past_32_bits(dims, layout):
    import torch
    import paper_2605_31500_amd as gt
    n, h, d = 1_100_001, 8, 256
    q = rows_of_bits(n, h * d, 3).view(n, h, d)
    pos = torch.rand((n, 3), device="cuda") * 100
    out = torch.empty_like(q)
    gt.gt_rope(pos, q, out, dims, layout=layout)
    t = slice(n - TAIL, n)
    want = torch.empty_like(q[t])
    gt.gt_rope(pos[t], q[t], want, dims, layout=layout)
    assert torch.equal(out[t], want)
    gt.gt_rope(pos, q, q, dims, layout=layout)
    assert torch.equal(out, q)


def test_diff_attention_past_32_bits():
    """The last rows refer to each other: as the same graph on them alone, up to
    the order of a row's sums (the small graph takes its rows otherwise)."""
    import torch
    import paper_2605_31500_amd as gt
    n, h, d = 550_001, 8, 256  # rows of 8 KB
    q, k, do = (rows_of_bits(n, 2 * h * d, s) for s in (5, 6, 7))
    v = torch.flip(k, (0,))
    rowptr, colidx = synth.ragged_graph(8, TAIL, max_deg=8, hubs={3: 300, 700: 900}, shuffle=True)
    rt, ct = synth.transpose_csr(rowptr, colidx, TAIL)
    lam = torch.linspace(0.1, 0.8, h, device="cuda")
    res = []
    for base in (0, n - TAIL):  # the tail's tensors alone, then the whole ones
        N = TAIL if base == 0 else n
        csr = []
        for rp, ci in ((rowptr, colidx), (rt, ct)):
            rp = np.concatenate([np.zeros(base, np.int64), rp])
            csr += [to_device(rp), to_device((ci + base).astype(np.int32))]
        t = [x[n - N:].view(N, 2 * h, d) for x in (q, k)] + [x[n - N:].view(N, h, 2 * d) for x in (v, do)]
        out, dv = torch.empty_like(t[2]), torch.empty_like(t[2])
        dq, dk, dl = torch.empty_like(t[0]), torch.empty_like(t[0]), torch.empty_like(lam)
        lse = torch.empty((N, 2 * h), device="cuda")
        gt.gt_diff_attn_fwd(csr[0], csr[1], t[0], t[1], t[2], lam, out, d ** -0.5, lse=lse)
        gt.gt_diff_attn_bwd(*csr, t[0], t[1], t[2], lam, t[3], lse, dq, dk, dv, dl, d ** -0.5)
        if base:
            for x in (out, dq, dk, dv):
                assert not torch.any(x[:base])
            assert bool(torch.all(torch.isneginf(lse[:base])))
        res.append([x[N - TAIL:].float().cpu().numpy() for x in (out, dq, dk, dv)] + [lse[N - TAIL:].cpu().numpy(), dl.cpu().numpy()])
        del out, dq, dk, dv
    for a, b in zip(*res):
        fin = np.isfinite(a)
        assert np.array_equal(fin, np.isfinite(b))
        a, b = np.where(fin, a, 0), np.where(fin, b, 0)
        # each value is rounded once to bf16, from sums that differ in fp32: by a step at most
        assert float(np.linalg.norm(a - b)) <= 2.0 ** -7 * float(np.linalg.norm(a))
