"""Operators of a training loop around the rows of a batch, as timed cases: rows looked up by the kind of an op with the
gradient of the table, a norm over the channels of each row with its gradients, and an AdamW step over many tensors with
its moments in 32 or in 8 bits.

Each case is one call (a step and the values that it leaves, where they are held in fewer bits) in a plain form of
elementary torch operations in 32 bits, or through the public binding.  Sizes are those of the repository's
configurations (128 and 256 columns, layer matrices of three blocks of rows, the 5.7 M rows of a batch of 4096 candidate
modules, the 474 k rows of a training batch) and generic ones: rows of some thousand channels, tables of 128 k kinds, some
hundred million parameters.
"""
import functools
import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
KEPT = 32                      # columns that share an exponent in kept rows
BLOCK = 128                    # places that share an exponent in 8-bit moments
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VALUES_MOST = 4096 * 1390 * 256   # of one array: a batch of 4096 modules of about 1390 nodes, 256 columns
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
SEED = 20240229                # of the draws by which 8-bit moments are rounded
STEPS = 400                    # done before the timed one


def listed():
    return [
        # the graph vector of one candidate: what an interactive caller waits for
        {"name": "norm_one_row", "do": "norm", "rows": 1, "C": 256, "dtype": "bf16", "act": "none"},
        # rows in front of a layer of a batch of candidate modules, the largest of this kind
        {"name": "norm_batch", "do": "norm", "rows": 4096 * 1390, "C": 256, "dtype": "bf16", "act": "silu"},
        # its gradients, with the one that goes past the norm
        {"name": "norm_back_batch", "do": "norm_back", "rows": 2000003, "C": 256, "dtype": "bf16", "act": "gelu", "kept": False, "past": True},
        # a training batch of fused-op samples whose inputs were kept in 8 bits
        {"name": "norm_back_kept", "do": "norm_back", "rows": 474011, "C": 256, "dtype": "f32", "act": "silu", "kept": True, "past": False},
        # wide rows of an odd width
        {"name": "norm_back_wide", "do": "norm_back", "rows": 8191, "C": 5003, "dtype": "f32", "act": "none", "kept": False, "past": True},
        # the vector of one op
        {"name": "embed_one_row", "do": "embed", "rows": 1, "C": 256, "kinds": 97, "dtype": "f32", "spread": "even", "padding": False},
        # the first features of a batch of candidate modules, by op kind
        {"name": "embed_batch", "do": "embed", "rows": 4096 * 1390, "C": 128, "kinds": 97, "dtype": "bf16", "spread": "skewed", "padding": False},
        # the table's gradient over a training batch: few kinds, very many rows of each
        {"name": "embed_back_kinds", "do": "embed_back", "rows": 474011, "C": 256, "kinds": 97, "dtype": "f32", "spread": "skewed", "padding": False},
        # a large table of an odd width: most kinds once or not at all, some very often, rows of padding
        {"name": "embed_back_table", "do": "embed_back", "rows": 65521, "C": 1031, "kinds": 128001, "dtype": "bf16", "spread": "skewed", "padding": True},
        # the parameters of an estimator of six layers of 256
        {"name": "adamw_estimator", "do": "adamw", "of": "estimator", "layers": 6, "width": 256, "p": "f32", "states": "f32"},
        # matrices in bf16 with their low halves, vectors in fp32
        {"name": "adamw_large", "do": "adamw", "of": "ragged", "tensors": 61, "total": 120000007, "pattern": 3, "p": "mixed", "states": "f32"},
        # the same with moments in 8 bits, the largest: a step and the values that it leaves
        {"name": "adamw_large_8bit", "do": "adamw", "of": "ragged", "tensors": 45, "total": 260000003, "pattern": 5, "p": "mixed", "states": "8bit"},
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(hi):
        # the configurations' widths, multiples of 16, or anything
        return rng.choice([rng.choice([128, 256]), 16 * log_int(1, hi // 16), log_int(16, hi)])
    do = rng.choice(["norm", "norm", "norm_back", "norm_back", "embed", "embed_back", "embed_back", "adamw", "adamw"])
    if do in ("norm", "norm_back"):
        dtype, C = rng.choice(["f32", "bf16"]), width(16384)
        most = VALUES_MOST // (2 if dtype == "bf16" else 4) // (1 if do == "norm" else 3) // max(C, 16)
        # ReLU's derivative jumps where the normalised value is zero: its gradient is not drawn over millions of values
        case = {"do": do, "rows": log_int(1, most), "C": C, "dtype": dtype, "act": rng.choice(["none", "relu", "silu", "gelu"] if do == "norm" else ["none", "silu", "gelu"])}
        if do == "norm_back":
            case.update(kept=rng.random() < 0.4, past=rng.random() < 0.5)
        return case
    if do in ("embed", "embed_back"):
        dtype, C = rng.choice(["f32", "bf16"]), width(8192)
        kinds = log_int(1, min(250000, VALUES_MOST // 8 // C))
        most = VALUES_MOST // (4 if dtype == "bf16" else 8) // max(C, 32)
        return {"do": do, "rows": log_int(1, most), "C": C, "kinds": kinds, "dtype": dtype, "spread": rng.choice(["even", "skewed", "skewed"]), "padding": rng.random() < 0.5}
    if rng.random() < 0.25:
        return {"do": do, "of": "estimator", "layers": rng.randint(1, 12), "width": 32 * rng.randint(1, 16), "p": rng.choice(["f32", "mixed"]), "states": rng.choice(["f32", "8bit"])}
    tensors = log_int(1, 250)
    return {"do": do, "of": "ragged", "tensors": tensors, "total": tensors * log_int(2, 40000000 // tensors), "pattern": rng.randint(0, 10 ** 6),
            "p": rng.choice(["f32", "bf16", "mixed"]), "states": rng.choice(["f32", "8bit", "8bit"])}


# ---- inputs ----
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 23)
    return g


def _tensors(case):
    """(elements, bf16 or not, decay or not) of every tensor, those in bf16 first; the same for every seed."""
    if case["of"] == "estimator":
        H, matrices, vectors = case["width"], [], []
        for layer in range(case["layers"]):
            matrices.append((96 if layer == 0 else 3 * H) * H)
            vectors += [H] if layer == 0 else [H, H, H]            # bias, and the norm's gamma and beta
        matrices += [H * H, H * H]
        vectors += [H, H, H, 1]
    else:
        r = random.Random(case["pattern"])
        size = [math.exp(2.5 * r.gauss(0, 1)) for _ in range(case["tensors"])]
        spare = case["total"] - case["tensors"]
        all_of = [1 + int(s * spare / sum(size)) for s in size]
        all_of[-1] += case["total"] - sum(all_of)
        matrices, vectors = [n for n in all_of if n >= 8192], [n for n in all_of if n < 8192]
    tensors = [(n, case["p"] != "f32", True) for n in matrices] + [(n, case["p"] == "bf16", False) for n in vectors]
    return [t for t in tensors if t[1]] + [t for t in tensors if not t[1]]


def _places(tensors):
    """Where each tensor begins among the state's places, places of the bf16 ones, and all."""
    at, total, half = [], 0, 0
    for n, bf16, _ in tensors:
        at.append(total)
        total += -(-n // BLOCK) * BLOCK
        half = total if bf16 else half
    return at, half, total


def _inputs(case, seed):
    """The tensors of a case in its storage types; the same for run and exact."""
    g = _gen(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)
    x = {}
    if case["do"] in ("norm", "norm_back"):
        rows, C, t = case["rows"], case["C"], TYPES[case["dtype"]]
        # a column has a size and an offset of its own, as activations have
        x["x"] = (normal(rows, C) * (0.5 + torch.rand(C, generator=g, device=DEV)) + normal(C)).to(t)
        x["gamma"], x["beta"] = 1 + 0.2 * normal(C), 0.2 * normal(C)
        if case["do"] == "norm_back":
            x["dy"] = normal(rows, C).to(t)
            x["past"] = normal(rows, C).to(t) if case["past"] else None
            if case["kept"]:
                x["code"], x["exponent"] = _keep(x.pop("x"))
            # the statistics that the forward pass left
            v = (_kept_values(x["code"], x["exponent"], C) if case["kept"] else x["x"]).float()
            x["mean"], x["rstd"] = _statistics(v)
    elif case["do"] in ("embed", "embed_back"):
        rows, C, kinds, t = case["rows"], case["C"], case["kinds"], TYPES[case["dtype"]]
        u = torch.rand(rows, generator=g, device=DEV, dtype=torch.float64)
        if case["spread"] == "skewed":                             # the k-th most frequent kind about as 1 / k
            rank = torch.floor(torch.exp(u * math.log(kinds + 1))) - 1
            order = torch.randperm(kinds, generator=g, device=DEV)
            x["id"] = order[rank.long().clamp(0, kinds - 1)].int()
        else:
            x["id"] = (u * kinds).long().clamp(0, kinds - 1).int()
        if case["padding"]:                                        # a tenth of the rows stands for nothing
            x["id"][torch.rand(rows, generator=g, device=DEV) < 0.1] = -1
        if case["do"] == "embed":
            x["table"] = normal(kinds, C).to(t)
        else:
            x["dy"] = normal(rows, C).to(t)
    else:
        tensors = _tensors(case)
        at, half, total = _places(tensors)
        used, size, decay = (torch.zeros(total, device=DEV) for _ in range(3))
        for a, (n, _, d) in zip(at, tensors):                      # gradients of a tensor have a size of their own
            used[a:a + n] = 1
            size[a:a + n] = 10.0 ** ((a // BLOCK) % 4 - 4)
            decay[a:a + n] = DECAY if d else 0.0
        w, grad = 0.05 * normal(total) * used, normal(total) * size
        m, v = 0.3 * normal(total) * size, (size * (0.3 + normal(total).abs())) ** 2 * used
        m = m * used
        x["p16"], x["low"] = _halves(w[:half])
        x["p32"], x["decay"] = w[half:].clone(), decay
        x["g16"], x["g32"] = (grad * used)[:half].bfloat16(), (grad * used)[half:].clone()
        if case["states"] == "8bit":
            x["m"], x["m_exponent"] = _codes(m.double(), 4, None)
            x["v"], x["v_exponent"] = _codes(v.double(), 5, None)
        else:
            x["m"], x["v"] = m, v
    return x


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if case["do"] == "adamw":
        s["t"] = torch.full((1,), STEPS, dtype=torch.int32, device=DEV)
    if own:
        s["ev"] = _evaluator()
        if case.get("kept"):
            s["kept"] = _binding().KeptRows(s["code"], s["exponent"], case["C"])
        if case["do"] == "adamw":
            tensors = _tensors(case)
            at, half, total = _places(tensors)
            params, s["grads"] = ([s[a + "16"][lo:lo + n] if bf16 else s[a + "32"][lo - half:lo - half + n] for lo, (n, bf16, _) in zip(at, tensors)] for a in "pg")
            o = s["opt"] = s["ev"].adamw(params, lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=[DECAY if d else 0.0 for _, _, d in tensors],
                                         states=case["states"], seed=SEED)
            # the state of a run that has gone on for a while
            o.m.copy_(s["m"])
            o.v.copy_(s["v"])
            o.steps[:1].copy_(s["t"])
            if half:
                o.low[:half].copy_(s["low"])
            if case["states"] == "8bit":
                o.m_exponent.copy_(s["m_exponent"])
                o.v_exponent.copy_(s["v_exponent"])
    return s


def _binding():
    from paper_2209_12769_amd import binding
    return binding


@functools.lru_cache(maxsize=None)
def _evaluator():
    return _binding().Evaluator(16, 32, 1, "f32", 1, 1, 1, device=DEV)


# ---- one pass ----
def run(s):
    return (_run_own if own else _run_plain)(s["case"], s)


def _scale(c):
    return math.sqrt(c["C"])


def _run_own(c, s):
    if c["do"] == "norm":
        y, mean, rstd = s["ev"].row_norm(s["x"], s["gamma"], s["beta"], eps=EPS, act=c["act"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["do"] == "norm_back":
        dx, dgamma, dbeta = s["ev"].row_norm_backward(s["dy"], s["kept"] if c["kept"] else s["x"], s["gamma"], s["beta"], s["mean"], s["rstd"],
                                                      act=c["act"], residual=s["past"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if c["do"] == "embed":
        return {"y": s["ev"].embed_rows(s["id"], s["table"], scale=_scale(c))}
    if c["do"] == "embed_back":
        return {"dtable": s["ev"].embed_rows_backward(s["dy"], s["id"], c["kinds"], scale=_scale(c))}
    s["opt"].step(s["grads"])
    out = {"p16": s["p16"], "p32": s["p32"]}
    if c["states"] == "8bit":
        out["w"], out["m"], out["v"] = s["opt"].values("wmv")
    else:
        out["m"], out["v"] = s["opt"].m, s["opt"].v
        if c["p"] != "f32":
            out["w"], = s["opt"].values("w")
    return out


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return (z > 0).to(z.dtype) if act == "relu" else torch.ones_like(z)


def _statistics(x):
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    return mean, 1 / torch.sqrt(var + EPS)


def _keep(x):
    """Rows kept in 8 bits: per row and 32 columns the smallest power of two 2^e of which 127 reach the largest value."""
    rows, C = x.shape
    nb = -(-C // KEPT)
    v = torch.zeros(rows, nb * KEPT, device=x.device)
    v[:, :C] = x
    v = v.view(rows, nb, KEPT)
    top = v.abs().amax(2)
    _, e = torch.frexp(top)
    e = e.int() - 7
    e = torch.clamp(e + (torch.ldexp(top, -e) > 127).int(), -126, 121)
    q = torch.clamp(torch.round(torch.ldexp(v, -e[..., None])), -127, 127)
    q = torch.where((q == 0) & (v != 0), torch.sign(v), q)
    return q.to(torch.int8).view(rows, nb * KEPT), (e + 127).to(torch.uint8)


def _kept_values(code, exponent, C):
    rows, nb = exponent.shape
    return torch.ldexp(code.view(rows, nb, KEPT).float(), exponent.int()[..., None] - 127).view(rows, nb * KEPT)[:, :C]


# An fp32 value as a bf16 number (halves round away from zero) and its low 16 bits; the two are the whole value.
def _halves(w):
    bits = w.contiguous().view(torch.int32)
    return ((bits + 0x8000) >> 16).to(torch.int16).view(torch.bfloat16), bits.to(torch.int16)


def _whole(p, low):
    low = low.int() & 0xFFFF
    hi = p.view(torch.int16).int() - ((low >= 0x8000) & ((p.view(torch.int16).int() & 0x7FFF) != 0)).int()
    return ((hi << 16) | low).view(torch.float32)


# 8-bit moments: per 128 places an exponent x, codes with 3 bits of mantissa and 4 (m, with a sign) or 5 (v) of exponent; a code's
# steps are 2^(x - 17) and 2^(x - 33) at the least, the largest value 1.875 2^x.  Rounded up by chance, in proportion: `u`, in
# units of a step, is added before the rest is cut off (to the nearest without it).  v is never rounded to zero.
def _least(bits):
    return 17 if bits == 4 else 33


def _pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _codes(a, bits, u):
    top = 8 * (1 << bits) - 1
    b = a.abs().view(-1, BLOCK)
    mant, e = torch.frexp(b.amax(1))                               # below 1; 1.875 2^x is 0.9375 2^(x + 1)
    x = torch.clamp(torch.where(b.amax(1) > 0, e - 1 + (mant > 0.9375).int(), -200), -126 if bits == 4 else -116, 127)
    y = (b * _pow2(_least(bits) - x)[:, None]).view(-1)       # in the least steps
    y = torch.where(y < 8, torch.round(y * 2.0 ** 20) * 2.0 ** -20, y)   # what fp32 keeps of them
    _, e = torch.frexp(y)
    shift = torch.clamp(e - 4, min=0)                              # 8 <= y / 2^shift < 16, or no shift
    n = torch.floor(y * _pow2(-shift) + (0.5 if u is None else u)).int() + 8 * shift
    n = torch.clamp(n, max=top)
    if bits == 5:
        n = torch.where((n == 0) & (b.view(-1) > 0), torch.ones_like(n), n)
    else:
        n = torch.where(a < 0, n + 128, n)
    return n.to(torch.uint8), (x + 127).to(torch.uint8)


def _code_values(code, exponent, bits):
    n = code.int() & (127 if bits == 4 else 255)
    e, mant = n >> 3, n & 7
    v = torch.where(e > 0, (8 + mant) * _pow2(e - 1), mant.double())
    v = (v.view(-1, BLOCK) * _pow2(exponent.int() - 127 - _least(bits))[:, None]).view(-1)
    return (torch.where(code > 127, -v, v) if bits == 4 else v).float()


def _mix(z):
    # the output function of splitmix64
    z = (z ^ ((z >> 30) & 0x3FFFFFFFF)) * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = (z ^ ((z >> 27) & 0x1FFFFFFFFF)) * (0x94D049BB133111EB - (1 << 64))
    return z ^ ((z >> 31) & 0x1FFFFFFFF)


def _chances(t, total):
    """16 bits for m and for v at every place: a draw for each two places."""
    key = _mix(SEED ^ _mix(t.long()))
    q = torch.arange(total // 2, device=DEV, dtype=torch.int64)
    r = _mix(key + q * (0xD1342543DE82EF95 - (1 << 64)))
    r = torch.stack([r & 0xFFFF, (r >> 16) & 0xFFFF, (r >> 32) & 0xFFFF, (r >> 48) & 0xFFFF], 1).view(-1, 2)
    return ((2 * r + 1).double() * 2.0 ** -17).unbind(1)


def _run_plain(c, s):
    if c["do"] == "norm":
        x = s["x"].float()
        mean, rstd = _statistics(x)
        y = _act((x - mean[:, None]) * rstd[:, None] * s["gamma"] + s["beta"], c["act"])
        return {"y": y.to(TYPES[c["dtype"]]), "mean": mean, "rstd": rstd}
    if c["do"] == "norm_back":
        x = _kept_values(s["code"], s["exponent"], c["C"]) if c["kept"] else s["x"].float()
        xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
        dz = s["dy"].float()
        if c["act"] != "none":
            dz = dz * _act_grad(xh * s["gamma"] + s["beta"], c["act"])
        u = dz * s["gamma"]
        dx = s["rstd"][:, None] * (u - u.mean(1)[:, None] - xh * (u * xh).mean(1)[:, None])
        if c["past"]:
            dx = dx + s["past"].float()
        return {"dx": dx.to(TYPES[c["dtype"]]), "dgamma": (dz * xh).sum(0, dtype=torch.float64).float(), "dbeta": dz.sum(0, dtype=torch.float64).float()}
    if c["do"] == "embed":
        y = s["table"][s["id"].long().clamp(min=0)].float() * _scale(c)
        return {"y": torch.where((s["id"] >= 0)[:, None], y, torch.zeros_like(y)).to(TYPES[c["dtype"]])}
    if c["do"] == "embed_back":
        # rows in the order of their kinds, differences of one running sum over them in 64 bits; rows of padding come first
        ids, order = torch.sort(s["id"], stable=True)
        ends = torch.searchsorted(ids, torch.arange(-1, c["kinds"], dtype=torch.int32, device=DEV), right=True)
        rows = s["dy"][order].t().contiguous()                     # along neighbours in memory: one scan a column
        sums = torch.nn.functional.pad(torch.cumsum(rows, 1, dtype=torch.float64), (1, 0))[:, ends]
        return {"dtable": ((sums[:, 1:] - sums[:, :-1]).t() * _scale(c)).to(TYPES[c["dtype"]]).contiguous()}
    # an AdamW step
    half, eight = s["p16"].numel(), c["states"] == "8bit"
    s["t"] += 1
    w, g = torch.cat([_whole(s["p16"], s["low"]), s["p32"]]), torch.cat([s["g16"].float(), s["g32"]])
    m = _code_values(s["m"], s["m_exponent"], 4) if eight else s["m"]
    v = _code_values(s["v"], s["v_exponent"], 5) if eight else s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    c1, c2 = ((1 - torch.pow(b, s["t"].double())).float() for b in (BETA1, BETA2))
    w = w - LR * ((m / c1) / (torch.sqrt(v / c2) + ADAM_EPS) + s["decay"] * w)
    if eight:
        um, uv = _chances(s["t"], m.numel())
        code, exponent = _codes(m.double(), 4, um)
        s["m"].copy_(code)
        s["m_exponent"].copy_(exponent)
        code, exponent = _codes(v.double(), 5, uv)
        s["v"].copy_(code)
        s["v_exponent"].copy_(exponent)
        m, v = _code_values(s["m"], s["m_exponent"], 4), _code_values(s["v"], s["v_exponent"], 5)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    p16, low = _halves(w[:half])
    s["p16"].copy_(p16)
    s["low"].copy_(low)
    s["p32"].copy_(w[half:])
    out = {"p16": s["p16"], "p32": s["p32"], "m": m, "v": v}
    if eight or c["p"] != "f32":
        out["w"] = w
    return out


# ---- what a pass cannot do without ----
def work(case):
    if case["do"] == "adamw":
        tensors = _tensors(case)
        total, half = sum(n for n, _, _ in tensors), sum(n for n, b, _ in tensors if b)
        per32, per16 = 4 + 4 + 4, 2 + 2 + 2 + 2 + 2                # the parameter, its gradient (and its low half)
        moments, values = (4, 12) if case["states"] == "8bit" else (16, 0 if case["p"] == "f32" else 4)
        return {"bytes": per16 * half + per32 * (total - half) + (moments + values) * total, "flops": 15 * total}
    b, rows, C = 4 if case["dtype"] == "f32" else 2, case["rows"], case["C"]
    if case["do"] == "norm":
        return {"bytes": 2 * b * rows * C + 8 * C + 8 * rows, "flops": 8 * rows * C}
    if case["do"] == "norm_back":
        x = 1 + 1 / KEPT if case["kept"] else b
        return {"bytes": (x + b * (3 if case["past"] else 2)) * rows * C + 16 * C + 8 * rows, "flops": 16 * rows * C}
    if case["do"] == "embed":
        return {"bytes": 4 * rows + b * C * (rows + min(rows, case["kinds"])), "flops": rows * C}
    return {"bytes": 4 * rows + b * C * (rows + case["kinds"]), "flops": rows * C}


# ---- the definitions in 64 bits ----
def exact(case, seed):
    x, f64 = _inputs(case, seed), torch.float64
    if case["do"] in ("norm", "norm_back"):
        C, act = case["C"], case["act"]
        normal = torch.distributions.Normal(torch.tensor(0.0, dtype=f64, device=DEV), torch.tensor(1.0, dtype=f64, device=DEV))
        gamma, beta = x["gamma"].double(), x["beta"].double()
        if case.get("kept"):
            scale = torch.pow(torch.tensor(2.0, dtype=f64, device=DEV), x["exponent"].double() - 127)
            v = (x["code"].double() * scale.repeat_interleave(KEPT, 1))[:, :C]
        else:
            v = x["x"].double()
        if case["do"] == "norm":
            var, mean = torch.var_mean(v, 1, correction=0)
            rstd = torch.rsqrt(var + EPS)
            z = torch.addcmul(beta, (v - mean.unsqueeze(1)).mul_(rstd.unsqueeze(1)), gamma)
            y = {"none": lambda: z, "relu": lambda: z * (z > 0), "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * normal.cdf(z)}[act]()
            return {"y": y, "mean": mean, "rstd": rstd}
        rstd = x["rstd"].double().unsqueeze(1)
        xh = (v - x["mean"].double().unsqueeze(1)) * rstd
        z = xh * gamma + beta
        dz = x["dy"].double()
        if act == "silu":
            dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        elif act == "gelu":
            dz = dz * (normal.cdf(z) + z * torch.exp(normal.log_prob(z)))
        elif act == "relu":
            dz = dz * (z > 0)
        u = dz * gamma
        dx = rstd * (u - u.sum(1, keepdim=True) / C - xh * ((u * xh).sum(1, keepdim=True) / C))
        if case["past"]:
            dx = dx + x["past"].double()
        return {"dx": dx, "dgamma": (dz * xh).sum(0), "dbeta": dz.sum(0)}
    if case["do"] == "embed":
        y = torch.nn.functional.pad(x["table"].double(), (0, 0, 0, 1)) * math.sqrt(case["C"])     # a row of zeros at the end
        return {"y": y[x["id"].long()]}
    if case["do"] == "embed_back":
        order = torch.argsort(x["id"], stable=True)
        order = order[x["id"][order] >= 0]
        ids = x["id"][order].long()
        out = torch.zeros(case["kinds"], case["C"], dtype=f64, device=DEV)
        count = torch.bincount(ids, minlength=case["kinds"])
        out[count > 0] = torch.segment_reduce(x["dy"][order].double(), "sum", lengths=count[count > 0], axis=0)
        return {"dtable": out * math.sqrt(case["C"])}
    # AdamW: moments in 8 bits are defined by operations in fp32, one rounding each
    half = x["p16"].numel()
    step32 = (lambda v: v.float().double()) if case["states"] == "8bit" else (lambda v: v)
    b1, b2, o1, o2 = (step32(torch.tensor(b, dtype=f64, device=DEV)) for b in (BETA1, BETA2, 1 - BETA1, 1 - BETA2))
    low = x["low"].long() % 65536
    hi = x["p16"].view(torch.int16).long() % 65536
    hi = torch.where((low >= 32768) & (hi % 32768 != 0), hi - 1, hi)
    bits = hi * 65536 + low
    w = torch.cat([torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int().view(torch.float32).double(), x["p32"].double()])
    g = torch.cat([x["g16"].double(), x["g32"].double()])
    m, v = x["m"].double(), x["v"].double()
    if case["states"] == "8bit":
        steps = torch.tensor([(8 + n % 8) * 2.0 ** (n // 8 - 1) if n >= 8 else float(n) for n in range(256)], dtype=f64, device=DEV)
        sign = 1 - 2 * (x["m"] >= 128).double()
        m = sign * steps[x["m"].long() % 128] * torch.exp2(x["m_exponent"].double() - 127 - 17).repeat_interleave(BLOCK)
        v = steps[x["v"].long()] * torch.exp2(x["v_exponent"].double() - 127 - 33).repeat_interleave(BLOCK)
    m = step32(step32(m * b1) + step32(g * o1))
    v = step32(step32(v * b2) + step32(step32(g * g) * o2))
    t = STEPS + 1
    step = m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
    w = w - LR * step - LR * x["decay"].double() * w
    if case["states"] == "8bit":
        def mix(z):
            z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) % 2 ** 64
            z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) % 2 ** 64
            return z ^ (z >> 31)
        key = mix(SEED ^ mix(t))
        z = torch.arange(m.numel() // 2, device=DEV) * (0xD1342543DE82EF95 - (1 << 64)) + (key - (1 << 64) if key >> 63 else key)
        z = (z ^ (z >> 30 & (1 << 34) - 1)) * (0xBF58476D1CE4E5B9 - (1 << 64))
        z = (z ^ (z >> 27 & (1 << 37) - 1)) * (0x94D049BB133111EB - (1 << 64))
        z = z ^ (z >> 31 & (1 << 33) - 1)

        def rounded(a, shift, least, most):
            r = torch.empty_like(a)
            r[0::2], r[1::2] = (z >> shift) % 65536, (z >> (shift + 32)) % 65536
            top = a.abs().view(-1, BLOCK).amax(1)
            x = torch.ceil(torch.log2(torch.clamp(top, min=1e-60) / 1.875)).clamp(-126 if least == 17 else -116, 127)
            x = torch.where(top <= 1.875 * torch.exp2(x - 1), x - 1, x).clamp(-126 if least == 17 else -116, 127)   # a logarithm rounded up
            unit = torch.exp2(x - least).repeat_interleave(BLOCK)
            y = a.abs() / unit
            y = torch.where(y < 8, torch.round(y * 2 ** 20) / 2 ** 20, y)
            step = torch.exp2((torch.floor(torch.log2(y.clamp(min=8))) - 3))
            step = torch.where(y >= 16 * step, 2 * step, step)
            n = torch.floor(y / step + (r + 0.5) / 65536) * step
            n = n.clamp(max=15 * 2.0 ** most)
            if least == 33:
                n = torch.where((n == 0) & (a > 0), torch.ones_like(n), n)
            return torch.sign(a) * n * unit
        m, v = rounded(m, 0, 17, 14), rounded(v, 16, 33, 30)
    out = {"p16": w[:half], "p32": w[half:], "m": m, "v": v}
    if case["states"] == "8bit" or case["p"] != "f32":
        out["w"] = w
    return out
