"""Performance cases of the operators around the sparse attention of a graph transformer's layer.

Three operators, each in both directions: differential attention over a CSR graph (the difference of two softmax maps
with a learned weight per head), rotary positions with several axes, and layer norm.  A case is one call.  With ``own``
false the operators are computed by elementary torch operations, with ``own`` true by this library's entry points.  The
graphs are of the families of this repository's named workloads (Erdos-Renyi, power law, R-MAT, lognormal hubs), each
row with its self-loop unless the case says otherwise, its sources distinct and sorted, made on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5  # of the layer norm
THETA = 10000.0  # of the rotary positions

# ------------------------------------------------------------------------------------------------------ the cases


def listed():
    return [
        # differential attention.  A molecule-sized batch or a sampled mini-batch: launches and latency
        _diff("diff-er2k-f32-1x32", "diff", "er", 2000, "f32", 1, 32, deg=8),
        # full-batch inference on a citation graph of 169 K papers, some of them without a reference (empty rows)
        _diff("diff-pl169k-f32-2x32", "diff", "powerlaw", 169343, "f32", 2, 32, exponent=2.1, loops=False),
        # the forward of a training step on a web or social graph with hubs, with the statistics of its backward
        _diff("diff-rmat1m-bf16-2x32-lse", "diff", "rmat", 1 << 20, "bf16", 2, 32, deg=24, lse=True),
        # a wide layer on a graph whose degrees vary by three orders of magnitude
        _diff("diff-lognormal200k-bf16-4x64", "diff", "lognormal", 200001, "bf16", 4, 64, deg=30),
        # its backward, on the citation graph and on a graph with hubs in bf16
        _diff("diffbwd-pl169k-f32-2x32", "diffbwd", "powerlaw", 169343, "f32", 2, 32, exponent=2.1),
        _diff("diffbwd-rmat500k-bf16-2x32", "diffbwd", "rmat", 500000, "bf16", 2, 32, deg=24),
        # rotary positions.  The gradient of the queries and keys of a sampled point cloud, real coordinates
        _rope("rope-inv-points16k-f32-4x32", 16381, "f32", 4, 32, "16,16", "pairs", "points", inverse=True),
        # the tokens of a long video on a (time, height, width) grid, queries and keys in one call
        _rope("rope-video1m-bf16-8x64", 1 << 20, "bf16", 8, 64, "16,24,24", "halves", "grid"),
        # layer norm.  The mini-batch's node states
        _norm("norm-2k-f32-128", "norm", 2000, "f32", 128),
        # a large graph's node states in a training step, with the statistics of the backward
        _norm("norm-1m-bf16-256", "norm", 1 << 20, "bf16", 256, stats=True),
        # its backward: the citation graph's hidden features, and a width that fits no vector load
        _norm("normbwd-169k-f32-512", "normbwd", 169343, "f32", 512),
        _norm("normbwd-60k-bf16-203", "normbwd", 60001, "bf16", 203),
    ]


def _diff(name, op, graph, n, dtype, h, d, **more):
    return _named(name, {"op": op, "graph": graph, "n": n, "dtype": dtype, "h": h, "d": d, **more})


def _rope(name, n, dtype, h, d, dims, layout, coords, inverse=False):
    return _named(name, {"op": "rope", "n": n, "dtype": dtype, "h": h, "d": d, "dims": dims, "layout": layout,
                         "coords": coords, "inverse": inverse, "both": True})


def _norm(name, op, n, dtype, f, stats=False):
    return _named(name, {"op": op, "n": n, "dtype": dtype, "f": f, "stats": stats, "affine": True})


def _named(name, c):
    if name:
        c["name"] = name
    return c


def _dims(c):
    return [int(x) for x in c["dims"].split(",")]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["diff", "diff", "diffbwd", "rope", "norm", "normbwd"])
        dtype = rng.choice(["f32", "bf16"])
        eb = 4 if dtype == "f32" else 2
        if op in ("diff", "diffbwd"):
            family = rng.choice(["er", "powerlaw", "rmat", "lognormal"])
            c = _diff(None, op, family, _log_int(rng, 1500, 1 << 20), dtype, rng.choice([1, 2, 4]),
                      rng.choice([32, 32, 64, 128]))
            if family == "powerlaw":
                c["exponent"] = round(rng.uniform(2.0, 2.6), 2)
            else:
                c["deg"] = rng.randint(4, 40)
            c["loops"] = rng.random() < 0.75
            c["lse"] = op == "diff" and rng.random() < 0.5
            row = 2 * c["h"] * c["d"]
            gathers = (2 if op == "diff" else 4) * c["n"] * _mean_degree(c) * row
            if c["n"] * _mean_degree(c) < 2.6e7 and gathers < (7e9 if op == "diff" else 6.5e9):
                return c
        elif op == "rope":
            h, d = rng.choice([1, 2, 4, 8]), rng.choice([32, 64, 128, 256])
            axes = rng.randint(1, 4)
            left, dims = d, []
            for a in range(axes):  # any even sizes that fit: the rest of the head passes through
                dims.append(2 * rng.randint(1, max(1, left // (2 * (axes - a)))))
                left -= dims[-1]
            c = _rope(None, _log_int(rng, 1000, 1 << 20), dtype, h, d, ",".join(map(str, dims)),
                      rng.choice(["pairs", "halves", "sections"]), rng.choice(["grid", "points"]), rng.random() < 0.4)
            c["both"] = rng.random() < 0.7
            if c["n"] * h * d * eb * (2 if c["both"] else 1) < 2.2e9:
                return c
        else:
            f = rng.choice([_log_int(rng, 8, 4096), 8 * _log_int(rng, 2, 512), rng.choice([64, 128, 256, 512, 1024])])
            c = _norm(None, op, _log_int(rng, 500, 1 << 20), dtype, f, stats=rng.random() < 0.5)
            c["affine"] = rng.random() < 0.8
            if c["n"] * f * eb * (1 if op == "norm" else 1.5) < 5.4e8:
                return c


# ----------------------------------------------------------------------------------------------------- the graphs

_KMAX, _SHIFT = 13000, 0.532  # the power law: P(k) ~ (k + shift)^-exponent, k = 1..kmax
_MU, _SIGMA = 2.5, 1.5  # the lognormal degrees, rescaled to the mean degree


def _mean_degree(c):
    """Entries per row, the self-loop among them."""
    loop = 1.0 if c.get("loops", True) else 0.0
    if c["graph"] == "powerlaw":
        top = min(_KMAX, c["n"] - 1)
        w = [(k + _SHIFT) ** -c["exponent"] for k in range(1, top + 1)]
        mean = sum(k * x for k, x in enumerate(w, 1)) / sum(w)
        return loop + (mean if loop else mean - 1)  # (without loops a row has one entry fewer: some have none)
    return float(c["deg"]) if c["graph"] == "rmat" else loop + c["deg"]


def _keys(c, g):
    """The graph's (row, source) pairs without its self-loops as row * n + source, repeats possible."""
    n, dev = c["n"], g.device

    def uniform_sources(rows):
        j = torch.randint(0, n - 1, rows.shape, generator=g, device=dev)
        return rows * n + j + (j >= rows)

    ids = torch.arange(n, device=dev)
    if c["graph"] == "er":
        return uniform_sources(ids.repeat_interleave(min(c["deg"], n - 1)))
    if c["graph"] == "powerlaw":
        k = torch.arange(1, min(_KMAX, n - 1) + 1, device=dev, dtype=torch.float64)
        cdf = torch.cumsum((k + _SHIFT) ** -c["exponent"], 0)
        u = torch.rand(n, generator=g, device=dev, dtype=torch.float64) * cdf[-1]
        deg = torch.searchsorted(cdf, u).clamp_(max=k.numel() - 1) + (1 if c.get("loops", True) else 0)
        return uniform_sources(ids.repeat_interleave(deg))
    if c["graph"] == "lognormal":
        x = torch.exp(_MU + _SIGMA * torch.randn(n, generator=g, device=dev, dtype=torch.float64)).clamp_(1, 200000)
        x *= c["deg"] * n / float(x.sum())
        deg = (x + torch.rand(n, generator=g, device=dev, dtype=torch.float64)).long().clamp_(1, n - 1)
        return uniform_sources(ids.repeat_interleave(deg))
    assert c["graph"] == "rmat"
    bits = (n - 1).bit_length()
    want = (c["deg"] - 1) * n
    src = torch.zeros(int(1.35 * want * 2 ** bits / n) + 64, dtype=torch.int64, device=dev)
    dst = torch.zeros_like(src)
    for _ in range(bits):  # quadrants with probabilities 0.57, 0.19, 0.19, 0.05
        u = torch.rand(src.shape, generator=g, device=dev)
        src = 2 * src + (u >= 0.76)
        dst = 2 * dst + (((u >= 0.57) & (u < 0.76)) | (u >= 0.95))
    ok = (src < n) & (dst < n) & (src != dst)
    perm = torch.randperm(n, generator=g, device=dev)
    keys = torch.unique(perm[dst[ok]] * n + perm[src[ok]])
    return keys[torch.randperm(keys.numel(), generator=g, device=dev)[:want]]


def _csr(keys, n):
    rows = keys // n
    rowptr = torch.zeros(n + 1, dtype=torch.int64, device=keys.device)
    rowptr[1:] = torch.cumsum(torch.bincount(rows, minlength=n), 0)
    return rowptr, (keys - rows * n).to(torch.int32)


# ----------------------------------------------------------------------------------------------------- the inputs


def _inputs(c, seed):
    """The call's inputs as tensors on the GPU, from the seed alone."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    n = c["n"]
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=dev) * std).to(dtype)

    s = {}
    if c["op"] in ("diff", "diffbwd"):
        h, d = c["h"], c["d"]
        keys = _keys(c, g)
        if c.get("loops", True):
            ids = torch.arange(n, device=dev)
            keys = torch.cat([keys, ids * n + ids])
        keys = torch.unique(keys)
        s["rowptr"], s["colidx"] = _csr(keys, n)
        if c["op"] == "diffbwd":
            s["rowptr_t"], s["colidx_t"] = _csr(torch.sort(keys % n * n + keys // n).values, n)
        std = 0.5 if 2 * h * d >= 512 else 1.0  # wide rows come from normalised layers
        s["Q"], s["K"] = normal(n, 2 * h, d, std=std), normal(n, 2 * h, d, std=std)
        s["V"] = normal(n, h, 2 * d, std=std)
        if c["op"] == "diffbwd":
            s["dout"] = normal(n, h, 2 * d, std=std)
        s["lam"] = 0.2 + 0.6 * torch.rand(h, generator=g, device=dev)
        s["scale"] = float(torch.tensor(d ** -0.5, dtype=torch.float32))
    elif c["op"] == "rope":
        h, d, axes = c["h"], c["d"], len(_dims(c))
        if c["coords"] == "grid":  # row-major in the axes, the last one fastest: sides of about n^(1/axes)
            side = max(2, round(n ** (1.0 / axes)))
            i = torch.arange(n, device=dev) + int(torch.randint(0, n, (1,), generator=g, device=dev))
            cols = []
            for _ in range(axes - 1):
                cols.append(i % side)
                i = i // side
            s["pos"] = torch.stack([i] + cols[::-1], 1).float().contiguous()
        else:  # points of a scan, in voxels
            s["pos"] = (torch.rand((n, axes), generator=g, device=dev) - 0.5) * 2000.0
        s["Q"] = normal(n, h, d)
        s["K"] = normal(n, h, d) if c["both"] else None
    else:
        f = c["f"]
        # node states: features with means of their own, rows of different norms
        x = torch.randn((n, f), generator=g, device=dev) + 0.5 * torch.randn(f, generator=g, device=dev)
        s["X"] = (x * torch.exp(0.4 * torch.randn((n, 1), generator=g, device=dev))).to(dtype)
        s["gamma"] = 1 + 0.2 * torch.randn(f, generator=g, device=dev) if c["affine"] else None
        s["beta"] = 0.2 * torch.randn(f, generator=g, device=dev) if c["affine"] else None
        if c["op"] == "normbwd":
            s["dout"] = normal(n, f)
    return s


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    s["case"] = c
    if c["op"] in ("diff", "diffbwd"):
        n, h = c["n"], c["h"]
        if c["op"] == "diff":
            s["out"] = torch.empty_like(s["V"])
            s["lse"] = torch.empty((n, 2 * h), device=s["Q"].device) if c.get("lse") else None
        else:
            # the forward's statistics, as a training step has them in hand
            s["lse"] = _maps_exact(s)[1].float()
            for k in "QKV":
                s["d" + k] = torch.empty_like(s[k])
            s["dlam"] = torch.empty_like(s["lam"])
    elif c["op"] == "rope":
        s["dims"] = _dims(c)
        s["outQ"] = torch.empty_like(s["Q"])
        s["outK"] = torch.empty_like(s["K"]) if c["both"] else None
    elif c["op"] == "norm":
        s["out"] = torch.empty_like(s["X"])
        s["mean"] = torch.empty(c["n"], device=s["X"].device) if c["stats"] else None
        s["rstd"] = torch.empty_like(s["mean"]) if c["stats"] else None
    else:
        x = s["X"].double()
        s["mean"] = x.mean(1).float()
        s["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt().float()
        s["dX"] = torch.empty_like(s["X"])
        s["dgamma"] = torch.empty(c["f"], device=x.device) if c["affine"] else None
        s["dbeta"] = torch.empty(c["f"], device=x.device) if c["affine"] else None
    return s


# ------------------------------------------------------------------------------------------------------- the calls


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2605_31500_amd as gt

    c = s["case"]
    if c["op"] == "diff":
        gt.gt_diff_attn_fwd(s["rowptr"], s["colidx"], s["Q"], s["K"], s["V"], s["lam"], s["out"], s["scale"],
                            lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]} if c.get("lse") else {"out": s["out"]}
    if c["op"] == "diffbwd":
        gt.gt_diff_attn_bwd(s["rowptr"], s["colidx"], s["rowptr_t"], s["colidx_t"], s["Q"], s["K"], s["V"], s["lam"],
                            s["dout"], s["lse"], s["dQ"], s["dK"], s["dV"], s["dlam"], s["scale"])
        return {k: s[k] for k in ("dQ", "dK", "dV", "dlam")}
    if c["op"] == "rope":
        gt.gt_rope(s["pos"], s["Q"], s["outQ"], s["dims"], K=s["K"], out_k=s["outK"], theta=THETA, layout=c["layout"],
                   inverse=c["inverse"])
        return {"Q": s["outQ"], "K": s["outK"]} if c["both"] else {"Q": s["outQ"]}
    if c["op"] == "norm":
        gt.gt_layernorm_fwd(s["X"], s["gamma"], s["beta"], s["out"], EPS, mean=s["mean"], rstd=s["rstd"])
        return {k: s[k] for k in ("out", "mean", "rstd") if s[k] is not None}
    gt.gt_layernorm_bwd(s["X"], s["dout"], s["gamma"], s["mean"], s["rstd"], s["dX"], dgamma=s["dgamma"],
                        dbeta=s["dbeta"])
    return {k: s[k] for k in ("dX", "dgamma", "dbeta") if s[k] is not None}


_GATHERED = 1 << 28  # values of gathered rows held at a time


def _pieces(e, width):
    """Ranges of entries, about _GATHERED gathered values each."""
    step = max(1, _GATHERED // width)
    return [(a, min(a + step, e)) for a in range(0, e, step)]


def _run_plain(s):
    c = s["case"]
    if c["op"] == "rope":
        return _rope_plain(s)
    if c["op"] == "norm":
        x = s["X"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        y = x * rstd[:, None]
        if c["affine"]:
            y = y * s["gamma"] + s["beta"]
        out = {"out": y.to(s["X"].dtype)}
        if c["stats"]:
            out.update(mean=mean, rstd=rstd)
        return out
    if c["op"] == "normbwd":
        dy = s["dout"].float()
        xhat = (s["X"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["gamma"] if c["affine"] else dy
        dx = g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)
        out = {"dX": (dx * s["rstd"][:, None]).to(s["X"].dtype)}
        if c["affine"]:  # (sums over all rows)
            out["dgamma"] = (dy * xhat).sum(0, dtype=torch.float64).float()
            out["dbeta"] = dy.sum(0, dtype=torch.float64).float()
        return out

    # differential attention
    h, d, n = c["h"], c["d"], c["n"]
    src = s["colidx"].long()
    dst = torch.repeat_interleave(torch.arange(n, device=src.device), s["rowptr"].diff(), output_size=src.numel())
    Q, K, V, lam = s["Q"], s["K"], s["V"], s["lam"]
    pieces = _pieces(src.numel(), 2 * h * d)
    w = torch.empty((src.numel(), 2 * h), device=src.device)
    for a, b in pieces:
        w[a:b] = (Q[dst[a:b]].float() * K[src[a:b]].float()).sum(-1) * s["scale"]
    if c["op"] == "diff":
        top = torch.full((n, 2 * h), -math.inf, device=src.device)
        top.scatter_reduce_(0, dst[:, None].expand(-1, 2 * h), w, "amax")
        w = torch.exp(w - top[dst])
        total = torch.zeros((n, 2 * h), device=src.device).index_add_(0, dst, w)
        w /= total[dst]
        w = w[:, 0::2] - lam * w[:, 1::2]
        out = torch.zeros((n, h, 2 * d), device=src.device)
        for a, b in pieces:
            out.index_add_(0, dst[a:b], w[a:b, :, None] * V[src[a:b]].float())
        res = {"out": out.to(V.dtype)}
        if c.get("lse"):
            res["lse"] = top + torch.log(total)
        return res
    dout = s["dout"]
    w = torch.exp(w - s["lse"][dst])
    ds = torch.empty_like(w)
    for a, b in pieces:
        ds[a:b] = (dout[dst[a:b]].float() * V[src[a:b]].float()).sum(-1).repeat_interleave(2, 1)
    delta = torch.zeros((n, 2 * h), device=src.device).index_add_(0, dst, w * ds)
    sign = torch.stack([torch.ones_like(lam), -lam], 1).reshape(-1)
    ds = sign * w * (ds - delta[dst]) * s["scale"]
    w = w[:, 0::2] - lam * w[:, 1::2]
    dQ = torch.zeros(Q.shape, device=src.device)
    dK, dV = torch.zeros_like(dQ), torch.zeros(V.shape, device=src.device)
    for a, b in pieces:
        i, j = dst[a:b], src[a:b]
        dQ.index_add_(0, i, ds[a:b, :, None] * K[j].float())
        dK.index_add_(0, j, ds[a:b, :, None] * Q[i].float())
        dV.index_add_(0, j, w[a:b, :, None] * dout[i].float())
    dlam = -delta[:, 1::2].sum(0, dtype=torch.float64).float()
    return {"dQ": dQ.to(Q.dtype), "dK": dK.to(Q.dtype), "dV": dV.to(Q.dtype), "dlam": dlam}


def _rope_pairs(dims, layout):
    """(first element, second element, axis, exponent of 1 / theta) of every rotated pair.  "pairs" and "halves": each
    axis has a section of the head with a spectrum of its own and turns neighbours, or the two halves of the section;
    "sections": one spectrum and two halves over all rotated elements, an axis has a stretch of the spectrum."""
    pairs, off, total = [], 0, sum(dims)
    for axis, width in enumerate(dims):
        for k in range(width // 2):
            if layout == "pairs":
                pairs.append((off + 2 * k, off + 2 * k + 1, axis, 2 * k / width))
            elif layout == "halves":
                pairs.append((off + k, off + width // 2 + k, axis, 2 * k / width))
            else:
                p = off // 2 + k
                pairs.append((p, total // 2 + p, axis, 2 * p / total))
        off += width
    return pairs


def _rope_plain(s):
    c = s["case"]
    dev = s["pos"].device
    lo, hi, axis, power = zip(*_rope_pairs(_dims(c), c["layout"]))
    lo, hi, axis = (torch.tensor(x, device=dev) for x in (lo, hi, axis))
    freq = torch.tensor([THETA ** -p for p in power], dtype=torch.float64, device=dev)
    # (the angle of a far position needs 64 bits)
    angle = s["pos"].double()[:, axis] * (-freq if c["inverse"] else freq)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turn(x):
        y = x.float()
        a, b = y[..., lo], y[..., hi]
        y[..., lo], y[..., hi] = a * cos - b * sin, a * sin + b * cos
        return y.to(x.dtype)

    # (a copy first: float() of a fp32 tensor is the tensor itself)
    out = {"Q": turn(s["Q"].clone())}
    if c["both"]:
        out["K"] = turn(s["K"].clone())
    return out


def work(case):
    c, n = case, case["n"]
    eb = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rope":
        both = 2 if c["both"] else 1
        return {"bytes": n * (4 * len(_dims(c)) + 2 * both * c["h"] * c["d"] * eb),
                "flops": 3 * n * both * c["h"] * sum(_dims(c))}
    if c["op"] == "norm":
        f = c["f"]
        return {"bytes": 2 * n * f * eb + (8 * n if c["stats"] else 0) + (8 * f if c["affine"] else 0),
                "flops": 8 * n * f}
    if c["op"] == "normbwd":
        f = c["f"]
        return {"bytes": 3 * n * f * eb + 8 * n + (12 * f if c["affine"] else 0), "flops": 14 * n * f}
    h, row = c["h"], 2 * c["h"] * c["d"]
    e = n * _mean_degree(c)
    csr = 8 * (n + 1) + 4 * e
    if c["op"] == "diff":  # scores, one sum for each map
        return {"bytes": csr + 4 * n * row * eb + (8 * n * h if c.get("lse") else 0) + 4 * h, "flops": 6 * e * row}
    # two dot products and three sums
    return {"bytes": 2 * csr + 7 * n * row * eb + 8 * n * h + 8 * h, "flops": 10 * e * row}


# --------------------------------------------------------------------------------------------------- in 64 bits


def _rows_of(s):
    n = s["rowptr"].numel() - 1
    return torch.searchsorted(s["rowptr"], torch.arange(s["colidx"].numel(), device=s["rowptr"].device), right=True) - 1, n


def _maps_exact(s):
    """Both maps' weights of every entry, [E, 2H], and their logarithms' sums per row, [N, 2H], in 64 bits."""
    dst, n = _rows_of(s)
    src = s["colidx"].long()
    maps, d = s["Q"].shape[1:]
    logit = torch.cat([torch.matmul(s["Q"][dst[a:b]].double().unsqueeze(2), s["K"][src[a:b]].double().unsqueeze(3))
                       .view(-1, maps) for a, b in _pieces(src.numel(), 2 * maps * d)]
                      or [torch.zeros((0, maps), dtype=torch.float64, device=src.device)]) * s["scale"]
    at = dst[:, None].expand(-1, maps)
    high = torch.full((n, maps), -math.inf, dtype=torch.float64, device=src.device)
    high = high.scatter_reduce(0, at, logit, "amax")
    total = torch.zeros_like(high).scatter_add(0, at, torch.exp(logit - high.gather(0, at)))
    lse = high + torch.log(total)
    return torch.exp(logit - lse.gather(0, at)), lse


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["op"] == "rope":
        pairs = _rope_pairs(_dims(c), c["layout"])
        coef = torch.zeros((len(_dims(c)), len(pairs)), dtype=torch.float64)
        first, second = [p[0] for p in pairs], [p[1] for p in pairs]
        for k, (_, _, axis, power) in enumerate(pairs):
            coef[axis, k] = math.exp(-power * math.log(THETA))
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=s["pos"].device),
                           torch.stack([(s["pos"].double() * coef[:, k].to(s["pos"].device)).sum(1)
                                        for k in range(len(pairs))], 1))
        if c["inverse"]:
            turn = turn.conj()

        def rotated(x):
            y = x.double()
            z = torch.complex(y[..., first], y[..., second]) * turn[:, None, :]
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y

        return {k: rotated(s[k]) for k in ("Q", "K") if s[k] is not None}
    if c["op"] in ("norm", "normbwd"):
        x = s["X"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False)
        if c["op"] == "norm":
            rstd = torch.rsqrt(var + EPS)
            y = (x - mean[:, None]) * rstd[:, None]
            if c["affine"]:
                y = torch.addcmul(s["beta"].double(), y, s["gamma"].double())
            return {"out": y, "mean": mean, "rstd": rstd} if c["stats"] else {"out": y}
        mean, rstd = mean.float().double(), torch.rsqrt(var + EPS).float().double()  # (the call's inputs)
        xhat = (x - mean[:, None]) * rstd[:, None]
        dy = s["dout"].double()
        g = dy * s["gamma"].double() if c["affine"] else dy
        f = c["f"]
        dx = rstd[:, None] / f * (f * g - g.sum(1, keepdim=True) - xhat * (g * xhat).sum(1, keepdim=True))
        if not c["affine"]:
            return {"dX": dx}
        return {"dX": dx, "dgamma": torch.einsum("nf,nf->f", dy, xhat), "dbeta": dy.sum(0)}

    h, d, n = c["h"], c["d"], c["n"]
    dst, _ = _rows_of(s)
    src = s["colidx"].long()
    p, lse = _maps_exact(s)
    lam = s["lam"].double()
    pieces = _pieces(src.numel(), 4 * h * d)

    def summed(at, values):
        total = torch.zeros((n, *values(0, 0).shape[1:]), dtype=torch.float64, device=src.device)
        for a, b in pieces:
            total.index_add_(0, at[a:b], values(a, b))
        return total

    mixed = p.view(-1, h, 2)[..., 0] - p.view(-1, h, 2)[..., 1] * lam
    if c["op"] == "diff":
        out = summed(dst, lambda a, b: mixed[a:b].unsqueeze(-1) * s["V"][src[a:b]].double())
        return {"out": out, "lse": lse} if c.get("lse") else {"out": out}
    p = torch.exp(torch.log(p) + (lse - lse.float().double())[dst])  # the weights by the statistics that the call has
    mixed = p.view(-1, h, 2)[..., 0] - p.view(-1, h, 2)[..., 1] * lam
    pv = torch.cat([(s["dout"][dst[a:b]].double() * s["V"][src[a:b]].double()).sum(-1) for a, b in pieces])
    pv = pv.unsqueeze(-1).expand(-1, h, 2).reshape(-1, 2 * h)
    mean = summed(dst, lambda a, b: p[a:b] * pv[a:b])
    grad = p * (pv - mean[dst]) * s["scale"]
    grad.view(-1, h, 2)[..., 1] *= -lam
    return {
        "dQ": summed(dst, lambda a, b: grad[a:b].unsqueeze(-1) * s["K"][src[a:b]].double()),
        "dK": summed(src, lambda a, b: grad[a:b].unsqueeze(-1) * s["Q"][dst[a:b]].double()),
        "dV": summed(src, lambda a, b: mixed[a:b].unsqueeze(-1) * s["dout"][dst[a:b]].double()),
        "dlam": -mean.view(n, h, 2)[..., 1].sum(0),
    }
