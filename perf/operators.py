"""Operators for deep estimators, as timed cases: a dense layer with bias, activation and residual, a norm over the
rows of each graph with an activation, rows kept in 8 bits for the backward pass, and the gradients of all.

Each case is one call (or the pair that belongs together: keep and restore) on rows of a graph batch, in a plain form
of elementary torch operations in 32 bits, or through the public binding.  Sizes are those of the repository's
configurations: 128 and 256 columns, layer matrices of three blocks of rows (own vector, two neighbour means),
the 5.7 M rows of a batch of 4096 candidate modules, the 53 k fused-op samples of a training batch.
"""
import functools
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
BLOCK = 32                     # columns that share an exponent in kept rows
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VALUES_MOST = 4096 * 1390 * 256   # of one array: a batch of 4096 modules of about 1390 nodes, 256 columns


def listed():
    return [
        # the graph vector of one candidate in the regression network: what an interactive caller waits for
        {"name": "dense_one_row", "do": "dense", "rows": 1, "K": 256, "N": 256, "dtype": "bf16", "act": "relu", "residual": False, "pre": False},
        # a layer of a search step: some hundred rows of an fp32 estimator
        {"name": "dense_search_step", "do": "dense", "rows": 437, "K": 384, "N": 128, "dtype": "f32", "act": "relu", "residual": False, "pre": False},
        # a residual layer of a large batch, the largest product
        {"name": "dense_layer", "do": "dense", "rows": 2000003, "K": 768, "N": 256, "dtype": "bf16", "act": "none", "residual": True, "pre": False},
        # a layer of widths that are no multiple of anything, with what its backward needs
        {"name": "dense_odd_widths", "do": "dense", "rows": 196311, "K": 201, "N": 139, "dtype": "f32", "act": "gelu", "residual": True, "pre": True},
        # gradients of a layer with a smooth activation on a bf16 batch
        {"name": "dense_back", "do": "dense_back", "rows": 524309, "K": 768, "N": 256, "dtype": "bf16", "act": "silu", "kept": False},
        # gradients of an fp32 layer whose inputs were kept in 8 bits: a training batch of fused-op samples
        {"name": "dense_back_kept", "do": "dense_back", "rows": 474011, "K": 384, "N": 128, "dtype": "f32", "act": "relu", "kept": True},
        # the norm in front of a layer, a batch of candidate modules
        {"name": "norm_modules", "do": "norm", "graphs": 4096, "mean_rows": 1390, "C": 256, "G": 8, "dtype": "bf16", "act": "silu"},
        # the same on one small module
        {"name": "norm_one_module", "do": "norm", "graphs": 1, "mean_rows": 729, "C": 128, "G": 4, "dtype": "f32", "act": "relu"},
        # its gradient on a training batch: very many graphs of a few rows, inputs kept in 8 bits
        {"name": "norm_back_samples", "do": "norm_back", "graphs": 52901, "mean_rows": 9, "C": 256, "G": 8, "dtype": "f32", "act": "silu", "kept": True},
        # and on a few large modules, as they are before fusion
        {"name": "norm_back_large_modules", "do": "norm_back", "graphs": 24, "mean_rows": 20011, "C": 256, "G": 8, "dtype": "bf16", "act": "gelu", "kept": False},
        # the activations of a layer of a training batch: kept and read back
        {"name": "keep_training_batch", "do": "keep", "rows": 474011, "K": 256, "dtype": "f32"},
        # the same for a handful of rows of an odd width
        {"name": "keep_few", "do": "keep", "rows": 1391, "K": 139, "dtype": "bf16"},
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):
        # the configurations' widths, multiples of 16, or anything
        return rng.choice([rng.choice([w for w in (128, 256) if lo <= w <= hi]), 16 * rng.randint(max(1, lo // 16), hi // 16), rng.randint(lo, hi)])
    do = rng.choice(["dense", "dense", "dense_back", "dense_back", "norm", "norm_back", "keep"])
    dtype = rng.choice(["f32", "bf16"])
    case = {"do": do, "dtype": dtype}
    if do in ("dense", "dense_back"):
        K, N = width(16, 768), width(16, 512)
        # fp32 products cost several times those in bf16
        most = min(VALUES_MOST // 4 // max(K, N), (400 if dtype == "bf16" else 60) * 10 ** 9 // (K * N))
        case.update(rows=log_int(1, most), K=K, N=N, act=rng.choice(["none", "relu", "gelu", "silu"]))
        if do == "dense":
            case.update(residual=rng.random() < 0.5, pre=rng.random() < 0.3)
        else:
            case.update(kept=rng.random() < 0.5)
    elif do in ("norm", "norm_back"):
        per = rng.choice([1, 4, 8, 16, 32, 32, rng.randint(2, 40)])
        G = max(1, min(rng.randint(1, 512) // per, 64))
        C = per * G
        most = VALUES_MOST // (2 if dtype == "bf16" else 4) // (1 if do == "norm" else 2) // C
        graphs = log_int(1, 65536)
        # ReLU's derivative jumps where the normalised value is zero: its gradient is not drawn over millions of values
        case.update(graphs=graphs, mean_rows=log_int(1, max(1, min(20000, most // graphs))), C=C, G=G,
                    act=rng.choice(["none", "relu", "silu", "gelu"] if do == "norm" else ["none", "silu", "gelu"]))
        if do == "norm_back":
            case.update(kept=rng.random() < 0.5)
    else:
        K = width(16, 768)
        case.update(rows=log_int(1, VALUES_MOST // 4 // K), K=K)
    return case


# ---- inputs ----
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    return g


def _offsets(case, seed):
    """Rows of each graph around the mean: some graphs without rows, some of one or two, the longest several times the
    mean; the same number of rows in all for every seed."""
    g = torch.Generator().manual_seed(seed * 31 + 5)
    n, mean = case["graphs"], case["mean_rows"]
    size = torch.exp(0.5 * torch.randn(n, generator=g, dtype=torch.float64))
    if n > 1:
        size[torch.rand(n, generator=g) < 0.01] = 0
        size[torch.rand(n, generator=g) < 0.01] = 1 / mean
    size[-1] = max(float(size[-1]), 1e-3)
    end = torch.cumsum(size, 0)
    off = torch.zeros(n + 1, dtype=torch.int64)
    off[1:] = torch.round(end * (n * mean / end[-1])).long()
    return off


def _inputs(case, seed):
    """The tensors of a case in its storage type; the same for run and exact."""
    g, t = _gen(seed), TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)
    x = {}
    if case["do"] in ("dense", "dense_back"):
        rows, K, N = case["rows"], case["K"], case["N"]
        x["x"] = torch.relu(normal(rows, K)).to(t)                      # activations of the layer before
        x["w"] = (normal(K, N) / math.sqrt(K)).to(t)
        x["b"] = 0.1 * normal(N)
        if case["do"] == "dense":
            x["r"] = normal(rows, N).to(t) if case["residual"] else None
        else:
            x["z"] = (normal(rows, N)).to(t) if case["act"] != "none" else None
            x["dy"] = (normal(rows, N) / math.sqrt(rows)).to(t)
    elif case["do"] in ("norm", "norm_back"):
        off, C = _offsets(case, seed), case["C"]
        rows = int(off[-1])
        x["off"] = off.to(device=DEV, dtype=torch.int32)
        # a column has a size and an offset of its own, as activations have
        x["x"] = (normal(rows, C) * (0.5 + torch.rand(C, generator=g, device=DEV)) + normal(C)).to(t)
        x["gamma"] = 1 + 0.2 * normal(C)
        x["beta"] = 0.2 * normal(C)
        if case["do"] == "norm_back":
            x["dy"] = normal(rows, C).to(t)
    else:
        size = torch.exp(2 * normal(1, case["K"]))                       # columns of very different size
        x["x"] = (normal(case["rows"], case["K"]).abs_() * size).to(t)
    if case.get("kept"):
        x["code"], x["exponent"] = _keep_plain(x.pop("x"))
    if case["do"] == "norm_back":
        # the statistics that the forward pass left
        src = _values(x["code"], x["exponent"], case["C"]) if case.get("kept") else x["x"]
        x["mean"], x["rstd"] = _statistics(src.float(), x["off"], case["G"])
    return x


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if own:
        state["ev"] = _evaluator()
        if case.get("kept"):
            state["kept"] = _binding().KeptRows(state["code"], state["exponent"], case["K"] if case["do"] == "dense_back" else case["C"])
    return state


def _binding():
    from paper_2209_12769_amd import binding
    return binding


@functools.lru_cache(maxsize=None)
def _evaluator():
    return _binding().Evaluator(16, 32, 1, "f32", 1, 1, 1, device=DEV)


# ---- one pass ----
def run(s):
    c = s["case"]
    return (_run_own if own else _run_plain)(c, s)


def _run_own(c, s):
    ev = s["ev"]
    if c["do"] == "dense":
        if c["pre"]:
            y, z = ev.dense(s["x"], s["w"], bias=s["b"], act=c["act"], residual=s["r"], want_pre=True)
            return {"y": y, "z": z}
        return {"y": ev.dense(s["x"], s["w"], bias=s["b"], act=c["act"], residual=s["r"])}
    if c["do"] == "dense_back":
        dx, dw, db = ev.dense_backward(s["dy"], s["kept"] if c["kept"] else s["x"], s["w"], act=c["act"], pre=s["z"])
        return {"dx": dx, "dw": dw, "db": db}
    if c["do"] == "norm":
        y, mean, rstd = ev.graph_norm(s["x"], s["off"], c["G"], s["gamma"], s["beta"], eps=EPS, act=c["act"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["do"] == "norm_back":
        dx, dgamma, dbeta = ev.graph_norm_backward(s["dy"], s["kept"] if c["kept"] else s["x"], s["off"], c["G"], s["gamma"],
                                                   s["beta"], s["mean"], s["rstd"], act=c["act"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    return {"x": ev.restore_rows(ev.keep_rows(s["x"]), dtype=s["x"].dtype)}


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _keep_plain(x):
    """Codes [rows, columns rounded up to 32] and exponent codes [rows, columns / 32]: a value is code * 2^(exponent - 127)."""
    rows, K = x.shape
    nb = -(-K // BLOCK)
    v = torch.zeros(rows, nb * BLOCK, device=x.device)
    v[:, :K] = x
    v = v.view(rows, nb, BLOCK)
    m = v.abs().amax(2)
    _, e = torch.frexp(m)                               # m = f 2^e, 0.5 <= f < 1
    e = e.int() - 7                                     # m <= 127 * 2^e unless f is above 127 / 128
    e = e + (torch.ldexp(m, -e) > 127).int()
    e = torch.clamp(e, -126, 121)
    finite = torch.isfinite(m)
    e = torch.where(finite & (m > 0), e, torch.full_like(e, -126))
    # two factors: 2^-e alone can pass the largest or fall under the smallest number
    h = torch.div(-e, 2, rounding_mode="floor")
    u = torch.ldexp(torch.ldexp(v, h[..., None]), (-e - h)[..., None])
    q = torch.clamp(torch.round(u), -127, 127)
    q = torch.where((q == 0) & (v != 0), torch.sign(v), q)
    q = torch.where(finite[..., None], q, torch.zeros_like(q))
    code = q.to(torch.int8).view(rows, nb * BLOCK)
    exponent = torch.where(finite, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return code, exponent


def _values(code, exponent, K):
    rows, nb = exponent.shape
    e = exponent.int() - 127
    v = torch.ldexp(code.view(rows, nb, BLOCK).float(), e[..., None])
    v = torch.where((exponent == 255)[..., None], torch.full_like(v, float("nan")), v)
    return v.view(rows, nb * BLOCK)[:, :K]


def _graph_of_row(off):
    sizes = (off[1:] - off[:-1]).long()
    return torch.repeat_interleave(torch.arange(sizes.numel(), device=off.device), sizes)


def _graph_sums(v, off):
    """Sums of [rows, groups] over the rows of each graph, in 64 bits: they run over up to millions of values.  As
    differences of one running sum over the groups, one after the other."""
    rows, G = v.shape
    run_ = torch.zeros(G * rows + 1, dtype=torch.float64, device=v.device)
    torch.cumsum(v.t().contiguous().view(-1), 0, dtype=torch.float64, out=run_[1:])
    at = off.long()[None, :] + rows * torch.arange(G, device=v.device)[:, None]
    return (run_[at[:, 1:]] - run_[at[:, :-1]]).t()


def _statistics(x, off, G):
    rows, C = x.shape
    gid = _graph_of_row(off)
    count = ((off[1:] - off[:-1]).double() * (C // G)).clamp(min=1)[:, None]
    x = x.view(rows, G, C // G)
    mean = (_graph_sums(x.sum(2), off) / count).float()
    var = _graph_sums(((x - mean[gid][..., None]) ** 2).sum(2), off) / count
    return mean.contiguous(), (1 / torch.sqrt(var + EPS)).float().contiguous()


def _run_plain(c, s):
    t = TYPES[c["dtype"]]
    if c["do"] == "dense":
        z = s["x"].float() @ s["w"].float() + s["b"]
        y = _act(z, c["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return {"y": y.to(t), "z": z.to(t)} if c["pre"] else {"y": y.to(t)}
    if c["do"] == "dense_back":
        x = _values(s["code"], s["exponent"], c["K"]) if c["kept"] else s["x"].float()
        dz = s["dy"].float()
        if c["act"] != "none":
            dz = dz * _act_grad(s["z"].float(), c["act"])
        return {"dx": (dz @ s["w"].float().t()).to(t), "dw": (x.t() @ dz).to(t), "db": dz.sum(0)}
    if c["do"] == "norm":
        x, off, G = s["x"].float(), s["off"], c["G"]
        rows, C = x.shape
        mean, rstd = _statistics(x, off, G)
        gid = _graph_of_row(off)
        z = ((x.view(rows, G, C // G) - mean[gid][..., None]) * rstd[gid][..., None]).view(rows, C) * s["gamma"] + s["beta"]
        return {"y": _act(z, c["act"]).to(t), "mean": mean, "rstd": rstd}
    if c["do"] == "norm_back":
        off, G = s["off"], c["G"]
        x = _values(s["code"], s["exponent"], c["C"]) if c["kept"] else s["x"].float()
        rows, C = x.shape
        gid = _graph_of_row(off)
        shape = (rows, G, C // G)
        xh = ((x.reshape(shape) - s["mean"][gid][..., None]) * s["rstd"][gid][..., None]).view(rows, C)
        dz = s["dy"].float()
        if c["act"] != "none":
            dz = dz * _act_grad(xh * s["gamma"] + s["beta"], c["act"])
        u = (dz * s["gamma"]).view(shape)
        count = ((off[1:] - off[:-1]).double() * (C // G)).clamp(min=1)[:, None]
        s1 = (_graph_sums(u.sum(2), off) / count).float()
        s2 = (_graph_sums((u * xh.view(shape)).sum(2), off) / count).float()
        dx = s["rstd"][gid][..., None] * (u - s1[gid][..., None] - xh.view(shape) * s2[gid][..., None])
        return {"dx": dx.view(rows, C).to(t), "dgamma": (dz * xh).sum(0), "dbeta": dz.sum(0)}
    code, exponent = _keep_plain(s["x"])
    return {"x": _values(code, exponent, c["K"]).to(t)}


# ---- what a pass cannot do without ----
def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    kept = 1 + 1 / BLOCK
    if case["do"] == "dense":
        rows, K, N = case["rows"], case["K"], case["N"]
        arrays = 1 + int(case["residual"]) + int(case["pre"])
        return {"bytes": b * (rows * (K + arrays * N) + K * N) + 4 * N, "flops": 2 * rows * K * N}
    if case["do"] == "dense_back":
        rows, K, N = case["rows"], case["K"], case["N"]
        reads = (kept if case["kept"] else b) * K + b * N * (1 if case["act"] == "none" else 2)
        return {"bytes": rows * (reads + b * K) + 2 * b * K * N + 4 * N, "flops": 4 * rows * K * N}
    if case["do"] in ("norm", "norm_back"):
        values = case["graphs"] * case["mean_rows"] * case["C"]
        small = 4 * (2 * case["C"] + 2 * case["graphs"] * case["G"] + case["graphs"])
        if case["do"] == "norm":
            return {"bytes": 2 * b * values + small, "flops": 8 * values}
        return {"bytes": ((kept if case["kept"] else b) + 2 * b) * values + small, "flops": 16 * values}
    return {"bytes": (2 * b + 2 * kept) * case["rows"] * case["K"], "flops": 4 * case["rows"] * case["K"]}


# ---- the definitions in 64 bits ----
def exact(case, seed):
    x = {k: (v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v) for k, v in _inputs(case, seed).items()}
    do, act = case["do"], case["act"] if "act" in case else "none"
    if case.get("kept"):
        K = case["K"] if do == "dense_back" else case["C"]
        # code * 2^(exponent - 127); nothing that is kept here is infinite
        scale = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=DEV), x["exponent"].double() - 127)
        x["x"] = (x["code"].double() * scale.repeat_interleave(BLOCK, 1))[:, :K]
    normal = torch.distributions.Normal(torch.tensor(0.0, dtype=torch.float64, device=DEV), torch.tensor(1.0, dtype=torch.float64, device=DEV))

    def f(z):
        return {"none": lambda: z, "relu": lambda: z * (z > 0), "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * normal.cdf(z)}[act]()

    def df(z):
        if act == "silu":
            return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        if act == "gelu":
            return normal.cdf(z) + z * torch.exp(normal.log_prob(z))
        return (z > 0).double() if act == "relu" else torch.ones_like(z)
    if do == "dense":
        z = torch.addmm(x["b"], x["x"], x["w"])
        y = f(z) if x["r"] is None else f(z) + x["r"]
        return {"y": y, "z": z} if case["pre"] else {"y": y}
    if do == "dense_back":
        dz = x["dy"] if x["z"] is None else x["dy"] * df(x["z"])
        return {"dx": torch.mm(dz, x["w"].t()), "dw": torch.mm(x["x"].t().contiguous(), dz), "db": dz.sum(0)}
    if do == "keep":
        # the value nearest to x among the multiples of the block's power of two, a multiple that is not zero if x is not
        rows, K = x["x"].shape
        out = torch.empty_like(x["x"])
        for c0 in range(0, K, BLOCK):
            v = x["x"][:, c0:c0 + BLOCK]
            m = v.abs().amax(1, keepdim=True)
            e = torch.ceil(torch.log2(m.clamp(min=1e-300) / 127)).clamp(-126, 121)
            e = torch.where((m > 0) & (m <= 127 * torch.exp2(e - 1)), e - 1, e).clamp(-126, 121)      # a logarithm rounded up
            step = torch.exp2(e)
            n = torch.round(v / step).clamp(-127, 127)
            n = torch.where((n == 0) & (v != 0), torch.sign(v), n)
            out[:, c0:c0 + BLOCK] = n * step
        return {"x": out}
    off, G, C = x["off"].long(), case["G"], case["C"]
    n, rows = off.numel() - 1, x["x"].shape[0]
    gid = torch.bucketize(torch.arange(rows, device=DEV), off[1:], right=True)

    def per_graph(v):
        return torch.zeros(n, G, dtype=torch.float64, device=DEV).index_add_(0, gid, v.reshape(rows, G, C // G).sum(2))

    def wide(v):
        return v[gid].repeat_interleave(C // G, 1)
    count = torch.clamp((off[1:] - off[:-1]) * (C // G), min=1).double().unsqueeze(1)
    if do == "norm":
        mean = per_graph(x["x"]) / count
        centred = x["x"] - wide(mean)
        rstd = torch.rsqrt(per_graph(centred * centred) / count + EPS)
        return {"y": f(centred * wide(rstd) * x["gamma"] + x["beta"]), "mean": mean, "rstd": rstd}
    xh = (x["x"] - wide(x["mean"])) * wide(x["rstd"])
    dz = x["dy"] * df(xh * x["gamma"] + x["beta"])
    u = dz * x["gamma"]
    dx = wide(x["rstd"]) * (u - wide(per_graph(u) / count) - xh * wide(per_graph(u * xh) / count))
    return {"dx": dx, "dgamma": (dz * xh).sum(0), "dbeta": dz.sum(0)}
