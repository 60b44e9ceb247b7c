"""Entry points of include/gt_layer.h without a GPU: the library exports what the
header declares, the header compiles as C, every refusal comes from the host
(no pointer is dereferenced, no kernel launched), and the binding refuses what
the library cannot see."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import paper_2605_31500_amd as gt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gt_layer.h")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
A = 0x100000  # never dereferenced: each call fails validation first
P, f32 = ctypes.c_void_p, ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    return gt.load_library()


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return set(re.findall(r"\b(gt_[a-z0-9_]+)\s*\(", text))


def test_exports_every_declared_symbol(lib):
    assert declared() == set(gt.LAYER_SYMBOLS)
    for n in declared():
        assert hasattr(lib, n), n


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not installed")
def test_header_compiles_as_c_and_links(tmp_path):
    src = tmp_path / "caller.c"
    src.write_text('#include <stdio.h>\n#include "gt_layer.h"\ntypedef void (*any_fn)(void);\nint main(void) {\n'
                   "    const any_fn fns[] = {%s};\n"
                   "    gt_rope_spec s = {1, {32, 0, 0, 0}, GT_ROPE_PAIRS, 0.0};\n"
                   "    for (unsigned i = 0; i < sizeof fns / sizeof fns[0]; ++i) if (!fns[i]) return 1;\n"
                   "    if (gt_rope(GT_DTYPE_F32, NULL, NULL, NULL, NULL, NULL, 4, 1, 32, &s, 0, NULL) != GT_ERROR_INVALID_VALUE) return 2;\n"
                   '    printf("%%zu\\n", sizeof s);\n    return 0;\n}\n'
                   % ", ".join("(any_fn)" + n for n in sorted(declared())))
    pkg, exe = os.path.join(ROOT, "paper_2605_31500_amd"), str(tmp_path / "caller")
    r = subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__", "-isystem",
                        os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), str(src), "-o", exe, "-L", pkg,
                        "-lgtattn", "-Wl,-rpath," + pkg, "-Wl,-rpath-link," + os.path.join(ROCM, "lib")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and int(r.stdout) == ctypes.sizeof(gt.GtRopeSpec), r.stdout + r.stderr


def diff_fwd(lib, dtype=0, rowptr=A, colidx=A, Q=A, K=2 * A, V=3 * A, lam=4 * A, out=5 * A, lse=6 * A, N=10, E=20, H=2, D=32,
             scale=0.1, tuning=None):
    return lib.gt_diff_attn_fwd(dtype, P(rowptr), P(colidx), P(Q), P(K), P(V), P(lam), P(out), P(lse), N, E, H, D, f32(scale),
                                tuning, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=5), 2), (dict(H=3), 2), (dict(H=16), 2), (dict(D=16), 2), (dict(D=48), 2), (dict(D=256), 2),
    (dict(D=512, dtype=1), 2), (dict(N=-1), 1), (dict(N=1 << 31), 1), (dict(E=-1), 1), (dict(E=1 << 31), 1), (dict(H=0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(rowptr=0), 1), (dict(colidx=0), 1),
    (dict(Q=0), 1), (dict(K=0), 1), (dict(V=0), 1), (dict(lam=0), 1), (dict(out=0), 1),
    (dict(K=2 * A + 8), 1), (dict(lam=4 * A + 2), 1), (dict(lse=6 * A + 2), 1),      # misaligned
    (dict(out=A), 1), (dict(out=3 * A + 16), 1), (dict(out=4 * A - 16), 1),          # out on Q, V, lambda
    (dict(lse=5 * A + 16), 1), (dict(lse=2 * A), 1),                                 # lse on out, K
    (dict(tuning=ctypes.byref(gt.GtTuning(chunk_edges=(1 << 31) - 1))), 1),
])
def test_diff_fwd_refusals(lib, kw, status):
    assert diff_fwd(lib, **kw) == status
    assert lib.gt_last_error_message()


def diff_bwd(lib, dtype=0, rowptr=A, colidx=A, rowptr_t=A, colidx_t=A, Q=A, K=2 * A, V=3 * A, lam=4 * A, dout=5 * A, lse=6 * A,
             dQ=7 * A, dK=8 * A, dV=9 * A, dlam=10 * A, N=10, E=20, H=2, D=32, scale=0.1):
    return lib.gt_diff_attn_bwd(dtype, P(rowptr), P(colidx), P(rowptr_t), P(colidx_t), P(Q), P(K), P(V), P(lam), P(dout), P(lse),
                                P(dQ), P(dK), P(dV), P(dlam), N, E, H, D, f32(scale), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=5), 2), (dict(H=3), 2), (dict(D=256), 2), (dict(N=-1), 1), (dict(E=-1), 1), (dict(scale=float("nan")), 1),
    (dict(rowptr_t=0), 1), (dict(colidx_t=0), 1), (dict(dout=0), 1), (dict(lse=0), 1), (dict(dQ=0), 1), (dict(dK=0), 1),
    (dict(dV=0), 1), (dict(dK=8 * A + 4), 1), (dict(dlam=10 * A + 1), 1),
    (dict(dQ=A), 1), (dict(dK=7 * A), 1), (dict(dV=8 * A + 16), 1), (dict(dV=5 * A), 1), (dict(dQ=6 * A), 1),
    (dict(dlam=4 * A), 1), (dict(dlam=9 * A), 1), (dict(N=0, dlam=10 * A + 1), 1),
])
def test_diff_bwd_refusals(lib, kw, status):
    assert diff_bwd(lib, **kw) == status
    assert lib.gt_last_error_message()


def rope(lib, dtype=0, pos=A, Q=2 * A, K=3 * A, outQ=4 * A, outK=5 * A, N=10, H=4, D=32, axes=2, dims=(16, 16), layout=0,
         theta=1e4, inverse=0, spec=True):
    s = gt.GtRopeSpec(axes, (ctypes.c_int32 * 4)(*dims), layout, theta)
    return lib.gt_rope(dtype, P(pos), P(Q), P(K), P(outQ), P(outK), N, H, D, ctypes.byref(s) if spec else None, inverse, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), 2), (dict(D=33), 2), (dict(D=514), 2), (dict(H=1024, D=128), 2), (dict(layout=3), 2), (dict(H=0), 1),
    (dict(N=-1), 1), (dict(N=1 << 31), 1), (dict(spec=False), 1), (dict(axes=0), 1), (dict(axes=5), 1),
    (dict(dims=(16, 18)), 1), (dict(dims=(15, 16)), 1), (dict(dims=(0, 16)), 1), (dict(dims=(-2, 16)), 1),
    (dict(dims=(1 << 30, 1 << 30)), 1), (dict(theta=0.0), 1), (dict(theta=-1.0), 1), (dict(theta=float("inf")), 1),
    (dict(theta=float("nan")), 1), (dict(pos=0), 1), (dict(Q=0), 1), (dict(outQ=0), 1), (dict(K=0), 1), (dict(outK=0), 1),
    (dict(pos=A + 2), 1), (dict(outQ=4 * A + 8), 1), (dict(outQ=2 * A + 16), 1), (dict(outQ=3 * A), 1), (dict(outK=2 * A), 1),
    (dict(outK=4 * A + 32), 1), (dict(outQ=A), 1), (dict(outK=3 * A + 16), 1),
])
def test_rope_refusals(lib, kw, status):
    assert rope(lib, **kw) == status
    assert lib.gt_last_error_message()


def norm_fwd(lib, dtype=0, X=A, gamma=2 * A, beta=3 * A, out=4 * A, mean=5 * A, rstd=6 * A, N=10, F=100, eps=1e-5):
    return lib.gt_layernorm_fwd(dtype, P(X), P(gamma), P(beta), P(out), P(mean), P(rstd), N, F, f32(eps), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), 2), (dict(F=16385), 2), (dict(F=0), 1), (dict(N=-1), 1), (dict(N=1 << 31), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(X=0), 1), (dict(out=0), 1), (dict(X=A + 4), 1),
    (dict(out=A + 16), 1), (dict(gamma=2 * A + 2), 1), (dict(mean=5 * A + 2), 1), (dict(out=2 * A), 1), (dict(mean=A), 1),
    (dict(mean=4 * A), 1), (dict(rstd=5 * A), 1), (dict(mean=3 * A), 1),
])
def test_norm_fwd_refusals(lib, kw, status):
    assert norm_fwd(lib, **kw) == status
    assert lib.gt_last_error_message()


def norm_bwd(lib, dtype=0, X=A, dout=2 * A, gamma=3 * A, mean=4 * A, rstd=5 * A, dX=6 * A, dgamma=7 * A, dbeta=8 * A, N=10, F=100):
    return lib.gt_layernorm_bwd(dtype, P(X), P(dout), P(gamma), P(mean), P(rstd), P(dX), P(dgamma), P(dbeta), N, F, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), 2), (dict(F=16385), 2), (dict(F=-3), 1), (dict(N=-1), 1), (dict(dout=0), 1), (dict(mean=0), 1),
    (dict(rstd=0), 1), (dict(dX=0), 1), (dict(dX=6 * A + 8), 1), (dict(dX=A + 16), 1), (dict(dX=2 * A + 16), 1),
    (dict(dX=3 * A), 1), (dict(dX=4 * A), 1), (dict(dgamma=6 * A), 1), (dict(dbeta=7 * A), 1), (dict(dgamma=3 * A), 1),
    (dict(dbeta=2 * A), 1), (dict(dgamma=7 * A + 1), 1),
])
def test_norm_bwd_refusals(lib, kw, status):
    assert norm_bwd(lib, **kw) == status
    assert lib.gt_last_error_message()


def test_empty_calls_enqueue_nothing(lib):
    assert diff_fwd(lib, N=0, E=0) == 0
    assert diff_bwd(lib, N=0, E=0, dlam=0) == 0
    assert rope(lib, N=0) == 0
    assert norm_fwd(lib, N=0) == 0
    assert norm_bwd(lib, N=0, dgamma=0, dbeta=0) == 0
    assert lib.gt_last_error_message() == b""


def test_binding_refuses_host_tensors():
    import torch
    z, i64, i32 = torch.zeros(3, 2, 32), torch.zeros(4, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)
    v, row = torch.zeros(3, 1, 64), torch.zeros(3, 8)
    with pytest.raises(ValueError, match="device"):
        gt.gt_diff_attn_fwd(i64, i32, z, z, v, torch.zeros(1), v, 0.1)
    with pytest.raises(ValueError, match="2H"):
        gt.gt_diff_attn_fwd(i64, i32, torch.zeros(3, 3, 32), z, v, torch.zeros(1), v, 0.1)
    with pytest.raises(ValueError, match="device"):
        gt.gt_diff_attn_bwd(i64, i32, i64, i32, z, z, v, torch.zeros(1), v, torch.zeros(3, 2), z, z, v, None, 0.1)
    with pytest.raises(ValueError, match="device"):
        gt.gt_rope(torch.zeros(3, 1), z, z, [32])
    with pytest.raises(ValueError, match="both"):
        gt.gt_rope(torch.zeros(3, 1), z, z, [32], K=z)
    with pytest.raises(ValueError, match="device"):
        gt.gt_layernorm_fwd(row, None, None, row)
    with pytest.raises(ValueError, match="N, F"):
        gt.gt_layernorm_fwd(z, None, None, z)
    with pytest.raises(ValueError, match="device"):
        gt.gt_layernorm_bwd(row, row, None, row[:, 0], row[:, 0], row)
