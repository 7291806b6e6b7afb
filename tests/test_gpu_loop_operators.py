"""What a training loop of one's own takes beside the dense layer: a norm over the channels of each row, rows by kind with the
table's gradient, and AdamW over many tensors, against plain implementations in 64 bits, element by element.

Tolerances count roundings.  U = 2^-24 is the most that rounding to fp32 is off by, relative to the value; R(t) =
finfo(t).eps / 2 the same for the storage type of an output.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def R(t):
    return torch.finfo(t).eps / 2


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2209_12769_amd import binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def ev(B):
    e = B.Evaluator(16, 32, 1, "f32", 1, 1, 1)
    yield e
    e.close()


def rand(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape))


def act(z, name):
    return {"none": lambda: z, "relu": lambda: torch.clamp(z, min=0), "silu": lambda: z * torch.sigmoid(z),
            "gelu": lambda: 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))}[name]()


def slope(z, name):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: s + z * s * (1 - s),
            "gelu": lambda: 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[name]()


def off_grid(x, ld, first):
    """x on the device, its rows `ld` elements apart, the first at element `first` of its buffer."""
    buf = torch.full((first + x.shape[0] * ld,), float("nan"), dtype=x.dtype, device="cuda:0")
    v = buf[first:first + x.shape[0] * ld].view(x.shape[0], ld)[:, :x.shape[1]]
    v.copy_(x)
    return v


def close(got, want, tol, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() / tol)[bad].max()), bad.nonzero()[:3].tolist())


# ---------------------------------------------------------------------------
# row norm
# ---------------------------------------------------------------------------
# a thread's values, a row's lanes, a workgroup's waves: the roundings of a sum over a row
D = 16 + 6 + 16


def norm_inputs(rows, C, dtype, seed=1):
    x = rand(seed, rows, C) * (0.5 + rand(seed + 1, C).abs()) + rand(seed + 2, C)
    return x.to(TYPES[dtype]), (1 + 0.3 * rand(seed + 3, C)).float(), (0.3 * rand(seed + 4, C)).float()


def norm_reference(x, gamma, beta, name, t):
    d = x.double()
    C = x.shape[1]
    mean = d.mean(1, keepdim=True)
    c = d - mean
    var = (c * c).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + EPS)
    # the sum over C is off by D roundings; what it lacks is found from the differences, off by D + 4 of their size
    m_off = (D + 2) * U * d.abs().mean(1, keepdim=True)
    size = c.abs().mean(1, keepdim=True) + m_off
    # less than a rounding of the differences' root mean square is not added
    e_mean = (D + 4) * U * size + U * torch.sqrt(var + m_off ** 2)
    # d = x - m squared and summed, less the square of what m lacks; both in units of the larger sum
    e_var = (D + 8) * U * (var + 2 * m_off ** 2)
    e_rstd = rstd * (0.5 * e_var / (var + EPS) + 4 * U)
    g, b = gamma.double(), beta.double()
    xh = c * rstd
    e_xh = rstd * (e_mean + U * (c.abs() + m_off)) + c.abs() * e_rstd + 2 * U * (xh.abs() + rstd * m_off)
    z = g * xh + b
    e_z = g.abs() * e_xh + U * z.abs()
    y = act(z, name)
    # slopes of the activations are below 1.13; their evaluation: eight roundings of the size of z
    e_y = (1.13 * e_z + 8 * U * z.abs() if name != "none" else e_z) + (R(t) + U) * y.abs()
    return (y, e_y), (mean[:, 0], (e_mean + U * mean.abs())[:, 0]), (rstd[:, 0], (e_rstd + U * rstd)[:, 0])


def check_norm(x, gamma, beta, name, t, got):
    for g, (want, tol), what in zip(got, norm_reference(x, gamma, beta, name, t), ("y", "mean", "rstd")):
        close(g, want, tol, what)


WIDTHS = [1, 2, 3, 7, 8, 9, 31, 64, 65, 100, 128, 255, 256, 257, 511, 512, 513, 768, 1000, 2048, 4099, 8192, 8193, 16383, 16384]
NAMES = ["none", "relu", "gelu", "silu"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("rows", [1, 3, 67])
def test_row_norm(ev, dtype, C, rows):
    t = TYPES[dtype]
    for name in NAMES if C in (7, 256, 513) else [NAMES[C % 4]]:
        x, gamma, beta = norm_inputs(rows, C, dtype)
        check_norm(x, gamma, beta, name, t, ev.row_norm(x.cuda(), gamma.cuda(), beta.cuda(), EPS, name))
    one = torch.ones(C), torch.zeros(C)
    check_norm(x, *one, "none", t, ev.row_norm(x.cuda(), eps=EPS))


# more rows than places for them, so that a place takes several
MANY = [(70001, 16), (300007, 1), (40003, 256), (20011, 100), (9001, 520), (3003, 1536), (1203, 9000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", MANY)
def test_row_norm_of_many_rows(ev, dtype, rows, C):
    x, gamma, beta = norm_inputs(rows, C, dtype)
    check_norm(x, gamma, beta, "silu", TYPES[dtype], ev.row_norm(x.cuda(), gamma.cuda(), beta.cuda(), EPS, "silu"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,first", [(0, 1), (3, 0), (8, 8), (1, 5)])
@pytest.mark.parametrize("C", [37, 256, 700])
def test_row_norm_rows_anywhere(ev, dtype, ld, first, C):
    """Rows apart and off every boundary, in place; what lies between rows is not touched."""
    t, rows = TYPES[dtype], 23
    x, gamma, beta = norm_inputs(rows, C, dtype)
    xv = off_grid(x, C + ld, first)
    got = ev.row_norm(xv, gamma.cuda(), beta.cuda(), EPS, "gelu", out=xv)
    check_norm(x, gamma, beta, "gelu", t, got)
    assert int(torch.isnan(xv._base.flatten()).sum()) == first + rows * ld


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,spread", [(1e5, 1.0), (1e6, 0.1), (-1e8, 8.0), (0.0, 1e-6), (3e12, 1e9)])
@pytest.mark.parametrize("C", [5, 200, 3000])
def test_row_norm_far_from_zero(ev, dtype, offset, spread, C):
    x = (offset + spread * rand(3, 40, C)).to(TYPES[dtype])
    one = torch.ones(C), torch.zeros(C)
    check_norm(x, *one, "none", TYPES[dtype], ev.row_norm(x.cuda(), eps=EPS))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("C", [40, 256, 600])
def test_row_norm_keeps_rows_apart(ev, dtype, bad, C):
    x, gamma, beta = norm_inputs(50, C, dtype)
    args = gamma.cuda(), beta.cuda(), EPS, "none"
    clean = ev.row_norm(x.cuda(), *args)
    x[7, C // 2] = bad
    got = ev.row_norm(x.cuda(), *args)
    fine = torch.arange(50) != 7
    for a, b in zip(got, clean):
        assert torch.equal(a[fine], b[fine])
    assert torch.isnan(got[0][7]).all() and torch.isnan(got[2][7])
    dy = rand(9, 50, C).to(TYPES[dtype]).cuda()
    dx = ev.row_norm_backward(dy, x.cuda(), *args[:2], *got[1:])[0]
    assert torch.equal(dx[fine], ev.row_norm_backward(dy, x.cuda(), *args[:2], *got[1:], out=torch.empty_like(dy))[0][fine])
    assert torch.isfinite(dx[fine]).all() and not torch.isfinite(dx[7]).any()


def norm_back_reference(x, dy, dres, gamma, beta, mean, rstd, name, t):
    g, b, m, r = gamma.double(), beta.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x.double() - m) * r
    e_xh = 3 * U * xh.abs()                               # the statistics are given: subtraction and product
    z = g * xh + b
    dz = dy.double() * slope(z, name)
    # the slopes' own slopes are below 1; evaluating one: sixteen roundings of size 1 + |z|
    e_dz = torch.zeros_like(dz) if name in ("none", "relu") else dy.double().abs() * (g.abs() * e_xh + 2 * U * (z.abs() + b.abs()) + 16 * U * (1 + z.abs()))
    e_dz = e_dz + U * dz.abs()
    u, e_u = g * dz, g.abs() * e_dz + U * (g * dz).abs()
    s1, s2 = u.mean(1, keepdim=True), (u * xh).mean(1, keepdim=True)
    e1 = (e_u + (D + 2) * U * u.abs()).mean(1, keepdim=True)
    e2 = (e_u * xh.abs() + u.abs() * e_xh + (D + 2) * U * (u * xh).abs()).mean(1, keepdim=True)
    dx = r * (u - s1 - xh * s2)
    e = r * (e_u + e1 + xh.abs() * e2 + e_xh * s2.abs() + 4 * U * (u.abs() + s1.abs() + (xh * s2).abs()))
    if dres is not None:
        dx = dx + dres.double()
        e = e + U * dx.abs()
    # 64 rows of a thread, then its runs, in fp32; then 64 bits twice, rounded each time
    n = min(64, x.shape[0]) + x.shape[0] / 64 + 6
    dgamma, dbeta = (dz * xh).sum(0), dz.sum(0)
    eg = (e_dz * xh.abs() + dz.abs() * e_xh).sum(0) + n * U * (dz * xh).abs().sum(0)
    eb = e_dz.sum(0) + n * U * dz.abs().sum(0)
    return (dx, e + (R(t) + U) * dx.abs()), (dgamma, eg), (dbeta, eb), z


def check_norm_back(ev, rows, C, dtype, name, kept, past, ld=None, first=0):
    t = TYPES[dtype]
    print(rows, C, dtype, name, kept, past, flush=True)
    x, gamma, beta = norm_inputs(rows, C, dtype)
    dy, dres = rand(11, rows, C).to(t), rand(12, rows, C).to(t) if past else None
    place = (lambda v: v.cuda()) if ld is None else (lambda v: off_grid(v, C + ld, first))
    xd = place(x)
    if kept:
        xd = ev.keep_rows(xd)
        x = ev.restore_rows(xd, torch.float32).cpu()
    c = x.double() - x.double().mean(1, keepdim=True)
    mean, rstd = x.double().mean(1).float(), (1 / torch.sqrt((c * c).mean(1) + EPS)).float()
    *want, z = norm_back_reference(x, dy, dres, gamma, beta, mean, rstd, name, t)
    if name == "relu":                                     # where z is next to zero the derivative may be either
        dy[z.abs() < 1e-4] = 0
        *want, z = norm_back_reference(x, dy, dres, gamma, beta, mean, rstd, name, t)
    rd = place(dres) if past else None
    got = ev.row_norm_backward(place(dy), xd, gamma.cuda(), beta.cuda(), mean.cuda(), rstd.cuda(), name, rd, out=rd if ld is not None else None)
    for g, (w, tol), what in zip(got, want, ("dx", "dgamma", "dbeta")):
        close(g, w, tol, what)
    if ld is not None and past:
        assert int(torch.isnan(rd._base.flatten()).sum()) == first + rows * ld


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("rows", [1, 3, 67])
def test_row_norm_backward(ev, dtype, C, rows):
    for k, name in enumerate(NAMES if C in (7, 256, 513, 16384) else [NAMES[C % 4]]):
        for kept in (False, True):
            check_norm_back(ev, rows, C, dtype, name, kept, (k + kept) % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", MANY)
@pytest.mark.parametrize("kept", [False, True])
def test_row_norm_backward_of_many_rows(ev, dtype, rows, C, kept):
    check_norm_back(ev, rows, C, dtype, "gelu" if kept else "silu", kept, not kept)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,first", [(0, 1), (3, 0), (8, 8), (1, 5)])
@pytest.mark.parametrize("C", [37, 256, 700])
def test_row_norm_backward_rows_anywhere(ev, dtype, ld, first, C):
    check_norm_back(ev, 23, C, dtype, "silu", False, True, ld, first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 37, 256, 700, 1031, 9001, 16384])
def test_row_norm_backward_in_place(ev, dtype, C):
    """The gradient of x in the place of what is read, which may be one tensor for all."""
    x, gamma, beta = (v.cuda() for v in norm_inputs(301, C, dtype))
    dy, dres = rand(11, 301, C).to(x.dtype).cuda(), rand(12, 301, C).to(x.dtype).cuda()
    _, mean, rstd = ev.row_norm(x, gamma, beta, EPS, "silu")
    for same in (False, True):
        past = dy if same else dres
        want = ev.row_norm_backward(dy, x, gamma, beta, mean, rstd, "silu", past)
        for k in range(2 if same else 3):
            a = [dy.clone(), x.clone(), past.clone()]
            if same:
                a[2] = a[0]
            got = ev.row_norm_backward(a[0], a[1], gamma, beta, mean, rstd, "silu", a[2], out=a[k])
            assert got[0] is a[k] and all(torch.equal(u, v) for u, v in zip(got, want)), (same, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_row_norm_without_rows(ev, dtype):
    x = torch.empty(0, 48, dtype=TYPES[dtype], device="cuda")
    y, mean, rstd = ev.row_norm(x)
    assert y.shape == (0, 48) and mean.shape == rstd.shape == (0,)
    dx, dgamma, dbeta = ev.row_norm_backward(x, x, None, None, mean, rstd)
    assert dx.shape == (0, 48) and not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("name", ["none", "gelu", "silu"])
def test_row_norm_gradients_against_differences(ev, name):
    """Central differences of sum(dy * y) along random directions of x, gamma and beta, in the fp32 kernel's own results:
    the difference of two sums of 64-bit products over 2 h, h = 2^-6."""
    rows, C, h = 9, 70, 2.0 ** -6
    x, gamma, beta = (v.double() for v in norm_inputs(rows, C, "f32"))
    dy = rand(21, rows, C)

    def y(x, gamma, beta):
        c = x - x.mean(1, keepdim=True)
        return act(gamma * c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) + beta, name)

    def loss(*v):
        return float((dy * ev.row_norm(v[0].float().cuda(), v[1].float().cuda(), v[2].float().cuda(), EPS, name)[0].double().cpu()).sum())
    _, mean, rstd = ev.row_norm(x.float().cuda(), gamma.float().cuda(), beta.float().cuda(), EPS, name)
    grads = ev.row_norm_backward(dy.float().cuda(), x.float().cuda(), gamma.float().cuda(), beta.float().cuda(), mean, rstd, name)
    for k, g in enumerate(grads):
        v = [x, gamma, beta]
        way = rand(30 + k, *v[k].shape)
        way = way / way.norm()
        up, down = ([w + s * h * way if i == k else w for i, w in enumerate(v)] for s in (1, -1))
        want = float((g.double().cpu() * way).sum())
        got = (loss(*up) - loss(*down)) / (2 * h)
        # the formula's own third-order term, from 64 bits, and the roundings of the two sums: 40 of each value's size
        third = abs((float((dy * y(*up)).sum()) - float((dy * y(*down)).sum())) / (2 * h) - want)
        assert third < 0.05 * max(1.0, abs(want))
        tol = third + 2 * 60 * U * float((dy.abs() * (y(*v).abs() + 1)).sum()) / (2 * h)
        assert abs(got - want) <= tol, (name, k, got, want, tol)


# ---------------------------------------------------------------------------
# rows by kind
# ---------------------------------------------------------------------------
def ids_of(rows, kinds, how, seed=5):
    r = np.random.default_rng(seed)
    if how == "even":
        k = r.integers(0, kinds, rows)
    elif how == "skewed":
        k = np.minimum(np.exp(r.random(rows) * math.log(kinds + 1)).astype(np.int64) - 1, kinds - 1)
    elif how == "one":
        k = np.full(rows, kinds // 2)
    elif how == "none":
        k = np.full(rows, -1)
    elif how == "sorted":
        k = np.sort(r.integers(0, kinds, rows))[::-1].copy()
    else:                                                  # a tenth stands for nothing
        k = np.where(r.random(rows) < 0.1, -1, r.integers(0, kinds, rows))
    return torch.from_numpy(k.astype(np.int32))


CHANNELS = [1, 3, 8, 17, 64, 139, 256, 520, 1031]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", CHANNELS + [4096, 8190, 65536])
@pytest.mark.parametrize("rows,kinds", [(1, 1), (1, 97), (5, 3), (1003, 97)])
def test_embed_rows(ev, dtype, C, rows, kinds):
    if rows * C > 5e6:
        rows = 37
    t = TYPES[dtype]
    table, ids = rand(1, kinds, C).to(t), ids_of(rows, kinds, "padding" if rows > 1 else "even")
    for scale in (1.0, math.sqrt(C), 0.0):
        want = table[ids.long().clamp(min=0)].float() * scale
        want[ids < 0] = 0
        got = ev.embed_rows(ids.cuda(), table.cuda(), scale)
        assert torch.equal(got.cpu(), want.to(t))          # one product, rounded once


def back_reference(dy, ids, kinds, scale, t):
    d = dy.double()
    on = ids >= 0
    want, size = (torch.zeros(kinds, d.shape[1], dtype=torch.float64).index_add_(0, ids[on].long(), v[on]) for v in (d, d.abs()))
    # 64 rows of a chunk, its four runs, three lists of chunks rounded to fp32 each; the scale as fp32 and its product
    s = abs(scale)
    return want * scale, (64 + 4 + 3) * U * s * size + (R(t) + 3 * U) * s * want.abs()


def check_embed_back(ev, rows, kinds, C, dtype, how, scale=0.7):
    t = TYPES[dtype]
    print(rows, kinds, C, dtype, how, flush=True)
    dy, ids = rand(2, rows, C).to(t), ids_of(rows, kinds, how)
    got = ev.embed_rows_backward(dy.cuda(), ids.cuda(), kinds, scale)
    close(got, *back_reference(dy, ids, kinds, scale, t), "dtable")
    assert torch.equal(got, ev.embed_rows_backward(dy.cuda(), ids.cuda(), kinds, scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("rows,kinds", [(1, 1), (1, 300), (2, 2), (15, 4), (16, 1), (17, 40), (300, 7), (1003, 97), (1003, 5000)])
def test_embed_rows_backward(ev, dtype, C, rows, kinds):
    for how in ("even", "padding", "skewed"):
        check_embed_back(ev, rows, kinds, C, dtype, how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["even", "skewed", "one", "none", "sorted", "padding"])
@pytest.mark.parametrize("rows,kinds,C", [(4096, 97, 40), (4097, 511, 8), (20011, 512, 24), (50021, 3, 16), (30011, 70001, 8), (262145, 300000, 4), (300007, 1, 3), (9001, 40, 700), (150001, 5, 264), (30011, 97, 2056), (70001, 3, 2056)])
def test_embed_rows_backward_of_many_rows(ev, dtype, how, rows, kinds, C):
    check_embed_back(ev, rows, kinds, C, dtype, how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,first", [(0, 1), (3, 0), (8, 8), (1, 5)])
@pytest.mark.parametrize("C", [37, 256, 700])
def test_embed_rows_anywhere(ev, dtype, ld, first, C):
    t, rows, kinds = TYPES[dtype], 230, 31
    table, ids, dy = rand(1, kinds, C).to(t), ids_of(rows, kinds, "padding"), rand(2, rows, C).to(t)
    y, dt = off_grid(torch.zeros(rows, C, dtype=t), C + ld, first), off_grid(torch.ones(kinds, C, dtype=t), C + ld, first)
    want = table[ids.long().clamp(min=0)].clone()
    want[ids < 0] = 0
    ev.embed_rows(ids.cuda(), off_grid(table, C + ld, first), out=y)
    assert torch.equal(y.cpu(), want)
    ev.embed_rows_backward(off_grid(dy, C + ld, first), ids.cuda(), kinds, 1.5, out=dt)
    close(dt, *back_reference(dy, ids, kinds, 1.5, t), "dtable")
    assert int(torch.isnan(y._base.flatten()).sum()) == first + rows * ld
    assert int(torch.isnan(dt._base.flatten()).sum()) == first + kinds * ld


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_embed_rows_reports_ids_out_of_range(B, ev, dtype):
    t, C, kinds = TYPES[dtype], 40, 9
    ids = torch.tensor([0, 8, 9, -2, 3, 2 ** 31 - 1, -2 ** 31, -1], dtype=torch.int32)
    inside = torch.where((ids >= 0) & (ids < kinds), ids, -1)
    table, dy = rand(1, kinds, C).to(t).cuda(), rand(2, 8, C).to(t).cuda()
    assert ev.check() == B.DC_OK
    y = ev.embed_rows(ids.cuda(), table)
    assert ev.check() == B.DC_ERR_INVALID_ARG and ev.check() == B.DC_OK
    assert torch.equal(y, ev.embed_rows(inside.cuda(), table)) and ev.check() == B.DC_OK
    d = ev.embed_rows_backward(dy, ids.cuda(), kinds)
    assert ev.check() == B.DC_ERR_INVALID_ARG
    assert torch.equal(d, ev.embed_rows_backward(dy, inside.cuda(), kinds)) and ev.check() == B.DC_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_embed_rows_backward_keeps_kinds_apart(ev, dtype, bad):
    rows, kinds, C = 5003, 211, 24
    dy, ids = rand(2, rows, C).to(TYPES[dtype]), ids_of(rows, kinds, "skewed")
    clean = ev.embed_rows_backward(dy.cuda(), ids.cuda(), kinds)
    dy[77, 3] = bad
    got = ev.embed_rows_backward(dy.cuda(), ids.cuda(), kinds)
    k = int(ids[77])
    assert not torch.isfinite(got[k, 3])
    got[k, 3] = clean[k, 3]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_embed_rows_without_rows(ev, dtype):
    ids, dy = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 48, dtype=TYPES[dtype], device="cuda")
    assert ev.embed_rows(ids, torch.ones(3, 48, dtype=TYPES[dtype], device="cuda")).shape == (0, 48)
    assert not ev.embed_rows_backward(dy, ids, 700).any()


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
f32 = np.float32
LISTS = {"one": [1], "small": [1, 7, 8, 9, 127, 128, 129, 0, 2047, 2048, 2049], "ragged": [5000, 1, 300, 40001, 16, 16385],
         "many": [1 + (k * 37) % 500 for k in range(250)]}


class Plain:
    """AdamW with its state in numpy, for tensors one behind the other at multiples of 128 places."""

    def __init__(self, params, decay, states, seed, lr, betas, eps):
        self.sizes, self.states, self.seed, self.t = [p.numel() for p in params], states, seed, 0
        self.lr, self.betas, self.eps = lr, betas, eps
        self.at = np.concatenate([[0], np.cumsum([-(-n // 128) * 128 for n in self.sizes])]).astype(np.int64)
        total = int(self.at[-1])
        self.w, self.m, self.v = np.zeros(total, f32), np.zeros(total, f32), np.zeros(total, f32)
        self.decay, self.mask = np.zeros(total), np.zeros(total, bool)
        for p, a, n, d in zip(params, self.at, self.sizes, decay):
            self.w[a:a + n], self.decay[a:a + n], self.mask[a:a + n] = p.double().cpu().numpy().reshape(-1), d, True
        self.mc = self.vc = self.me = self.ve = None
        self.first = 0                                     # the state's place that these begin at

    def flat(self, grads):
        g = np.zeros(self.w.size, f32)
        for x, a, n in zip(grads, self.at, self.sizes):
            g[a:a + n] = x.double().cpu().numpy().reshape(-1)
        return g

    def step(self, grads, scale=1.0):
        self.t += 1
        b1, b2 = self.betas
        g = self.flat(grads) * f32(scale)
        m, v, w = self.m, self.v, self.w.astype(np.float64)
        # operations of fp32, rounded one by one
        m = m * f32(b1) + g * f32(1 - b1)
        v = v * f32(b2) + (g * g) * f32(1 - b2)
        m64, v64 = m.astype(np.float64), v.astype(np.float64)
        step = m64 / (1 - b1 ** self.t) / (np.sqrt(v64 / (1 - b2 ** self.t)) + self.eps)
        new = w - self.lr * (step + self.decay * w)
        # six roundings of the quotient (the two corrections, both products, root, sum, quotient) and those of the sum;
        # lr, decay and eps are rounded to fp32 too
        self.tol = 2 * U * np.abs(w) + self.lr * (12 * np.abs(step) + 4 * self.decay * np.abs(w)) * U + U * np.abs(new)
        self.want = new
        self.w = new.astype(f32)
        if self.states == "8bit":
            self.mc, self.me, self.m = self.codes(m, True)
            self.vc, self.ve, self.v = self.codes(v, False)
        else:
            self.m, self.v = m, v

    def chances(self):
        def mix(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            return z ^ (z >> np.uint64(31))
        with np.errstate(over="ignore"):
            key = mix(np.array([self.seed], np.uint64) ^ mix(np.array([self.t], np.uint64)))
            r = mix(key + (self.first // 2 + np.arange(self.w.size // 2, dtype=np.uint64)) * np.uint64(0xD1342543DE82EF95))
        return r.view(np.uint16).reshape(-1, 2)[:, 0], r.view(np.uint16).reshape(-1, 2)[:, 1]

    def codes(self, a, is_m):
        """(codes, exponent bytes, values): by the numbers themselves, not their bits."""
        r = self.chances()[0 if is_m else 1].astype(np.float64)
        least, top, low = (17, 127, -126) if is_m else (33, 255, -116)
        size = np.abs(a.astype(np.float64)).reshape(-1, 128)
        most = size.max(1)
        with np.errstate(divide="ignore", invalid="ignore"):
            x = np.where(most > 0, np.ceil(np.log2(most / 1.875)), -1000)
        x = np.where(most > np.ldexp(1.875, np.clip(x, -200, 200).astype(int)), x + 1, x)
        x = np.where((most > 0) & (most <= np.ldexp(1.875, np.clip(x - 1, -200, 200).astype(int))), x - 1, x)
        bad = ~np.isfinite(most)
        x = np.where(bad, 0, np.clip(x, low, 127)).astype(int)
        y = np.where(bad[:, None], 0, size * np.ldexp(1.0, least - x)[:, None]).reshape(-1)      # in the least steps
        y = np.where(y < 8, np.rint(y * 2 ** 20) / 2 ** 20, y)       # as far as fp32 goes there
        k = np.maximum(np.floor(np.log2(np.maximum(y, 1))) - 3, 0).astype(int)
        n = np.floor(y / np.ldexp(1.0, k) + (2 * r + 1) / 2 ** 17).astype(int) + 8 * k
        n = np.minimum(n, top)
        if not is_m:
            n = np.where((n == 0) & (a > 0), 1, n)
        n = np.where(np.repeat(bad, 128), 0, n)
        f, e = n & 7, n >> 3
        value = np.where(e > 0, np.ldexp(8.0 + f, np.maximum(e - 1, 0)), f) * np.repeat(np.ldexp(1.0, x - least), 128)
        value = np.where(np.repeat(bad, 128), np.nan, value)
        if is_m:
            sign = np.signbit(a) & ~np.repeat(bad, 128)
            n, value = np.where(sign, n | 128, n), np.where(np.signbit(a), -value, value)
        return n.astype(np.uint8), np.where(bad, 255, x + 127).astype(np.uint8), value.astype(f32)


def tensors_of(sizes, p, seed=1):
    kinds = {"f32": ["f32"], "bf16": ["bf16"], "mixed": ["bf16", "f32", "f32"]}[p]
    return [(0.1 * rand(seed + k, n)).to(TYPES[kinds[k % len(kinds)]]).cuda() for k, n in enumerate(sizes)]


def grads_of(params, k, g="own"):
    sizes = [10.0 ** (-(i % 5)) for i in range(len(params))]
    return [(s * rand(1000 * k + i, p.numel())).to(p.dtype if g == "own" else TYPES[g]).cuda().view(p.shape) for i, (p, s) in enumerate(zip(params, sizes))]


def check_state(o, plain, params):
    """The step's results against the plain ones, which then go on from the kernel's own w."""
    w, m, v = (x.cpu().numpy() for x in o.values("wmv"))
    assert not w[~plain.mask].any() and not m[~plain.mask].any() and not v[~plain.mask].any()
    bad = ~(np.abs(w.astype(np.float64) - plain.want) <= plain.tol)
    assert not bad[plain.mask].any(), (int(bad.sum()), (np.abs(w - plain.want) / plain.tol)[bad][:3], np.flatnonzero(bad)[:3])
    assert np.array_equal(m, plain.m, equal_nan=True) and np.array_equal(v, plain.v, equal_nan=True)
    if o.states == "8bit":
        on = plain.mask
        assert np.array_equal(o.m.cpu().numpy()[on], plain.mc[on]) and np.array_equal(o.v.cpu().numpy()[on], plain.vc[on])
        assert np.array_equal(o.m_exponent.cpu().numpy(), plain.me) and np.array_equal(o.v_exponent.cpu().numpy(), plain.ve)
    for p, a in zip(params, o.at):
        mine = torch.from_numpy(w[a:a + p.numel()])
        p = p.flatten().cpu()
        if p.dtype == torch.float32:
            assert torch.equal(p, mine)
        elif p.numel():                                    # halves away from zero
            bits = mine.view(torch.int32).numpy().astype(np.int64) & 0xFFFFFFFF
            assert np.array_equal(p.view(torch.int16).numpy().astype(np.int64) & 0xFFFF, (bits + 0x8000) >> 16 & 0xFFFF)
    assert o.steps.tolist() == [plain.t, 0]
    plain.w = w


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("p", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", list(LISTS))
@pytest.mark.parametrize("g", ["own", "f32", "bf16"])
def test_adamw(ev, states, p, sizes, g):
    params = tensors_of(LISTS[sizes], p)
    decay = [0.1 * (k % 3) for k in range(len(params))]
    args = dict(lr=3e-3, betas=(0.9, 0.98), eps=1e-7)
    o, plain = ev.adamw(params, **args, weight_decay=decay, states=states, seed=2 ** 63 + 11), Plain(params, decay, states, 2 ** 63 + 11, **args)
    for k in range(3):
        grads = grads_of(params, k, g)
        o.step(grads)
        plain.step(grads)
        check_state(o, plain, params)


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("sizes", [[2048 * 3], [2048 * 4], [2048 * 4, 1], [2048 * 2047, 2048], [2048 * 2047, 2048, 1], [2048 * 2046 + 1] * 2])
def test_adamw_of_whole_chunks(ev, states, sizes):
    """Around the sizes at which workgroups are full and calls are small."""
    params = tensors_of(sizes, "mixed")
    args = dict(lr=3e-3, betas=(0.9, 0.98), eps=1e-7)
    o, plain = ev.adamw(params, **args, weight_decay=0.1, states=states, seed=3), Plain(params, [0.1] * len(sizes), states, 3, **args)
    for k in range(2):
        grads = grads_of(params, k)
        o.step(grads)
        plain.step(grads)
        check_state(o, plain, params)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_adamw_of_nothing(ev, states):
    """A step without elements is one all the same."""
    none = torch.zeros(0, device="cuda")
    for params, grads in [([], []), ([none], [none]), (tensors_of([300, 2049], "mixed"), [None, None]), ([none] * 100, [none] * 100)]:
        was = [p.clone() for p in params]
        o = ev.adamw(params, states=states)
        for _ in range(3):
            o.step(grads)
        assert o.steps.tolist() == [3, 0] and all(torch.equal(a, b) for a, b in zip(was, params))
        w, m, v = o.values()
        assert w.numel() == o.total and not m.any() and not v.any()


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("first", [1, 3, 8])
def test_adamw_of_parts_of_a_buffer(ev, states, first):
    """Parameters and gradients off every boundary, between others that stay as they are; gradients times a device number."""
    sizes = [1, 300, 2050, 77]
    bufs, params, grads = [], [], []
    for k, n in enumerate(sizes):
        for to, t in ((params, TYPES["bf16" if k % 2 else "f32"]), (grads, TYPES["f32" if k % 2 else "bf16"])):
            b = torch.full((n + 2 * first,), 7.0, dtype=t, device="cuda")
            bufs.append((b, n))
            to.append(b[first:first + n])
            to[-1].copy_(rand(50 + len(bufs), n))
    args = dict(lr=1e-2, betas=(0.8, 0.9), eps=1e-8)
    o, plain = ev.adamw(params, **args, weight_decay=0.05, states=states), Plain(params, [0.05] * 4, states, 0, **args)
    scale = torch.tensor([0.3], device="cuda")
    for _ in range(2):
        o.step(grads, scale)
        plain.step(grads, 0.3)
        check_state(o, plain, params)
    for b, n in bufs:
        assert (b[:first] == 7).all() and (b[first + n:] == 7).all()


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_adamw_leaves_tensors_without_a_gradient(ev, states):
    params = tensors_of([300, 200, 100], "mixed")
    o = ev.adamw(params, states=states)
    o.step(grads_of(params, 0))
    before = [p.clone() for p in params] + [x.clone() for x in o.values()]
    g = grads_of(params, 1)
    o.step([g[0], None, g[2]])
    after = o.values()
    assert torch.equal(params[1], before[1]) and not torch.equal(params[0], before[0])
    for x, y in zip(after, before[3:]):
        assert torch.equal(x[384:640], y[384:640]) and not torch.equal(x[:300], y[:300])
    o.step([None] * 3)
    assert o.steps.tolist() == [3, 0] and torch.equal(o.values("w")[0], after[0])
    empty = ev.adamw([], states=states)
    empty.step([])
    assert empty.steps.tolist() == [1, 0] and empty.values("m")[0].shape == (0,)


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("eps", [1e-8, 1.1e-10, 0.9e-10, 1e-30])
@pytest.mark.parametrize("values", ["zeros", "wide", "edges", "bad"])
def test_adamw_of_unusual_gradients(ev, states, values, eps):
    n = 128 * 6
    r = np.random.default_rng(3)
    with np.errstate(over="ignore"):
        g = {"zeros": np.zeros(n), "wide": np.exp(r.uniform(-100, 40, n)) * r.choice([-1, 1], n),
             # v from the least to the largest, blocks whose largest value is a code's or just above
             "edges": np.concatenate([np.full(128, 1e-22), np.full(128, 1.8e19), [1e19] + [1e-15] * 127, np.geomspace(1e-20, 1, 128), [-1.875] + [1.0] * 127, [1.8750001] + [2.0 ** -k for k in range(127)]]),
             "bad": np.concatenate([[np.nan] + [1.0] * 127, [np.inf] + [1.0] * 127, [-np.inf] + [2.0] * 127, np.full(128, 3e38), np.full(128, 1e20), np.ones(128)])}[values].astype(f32)
    params = tensors_of([n], "f32")
    args = dict(lr=1e-3, betas=(0.9, 0.999), eps=eps)
    o, plain = ev.adamw(params, **args, weight_decay=0.0, states=states), Plain(params, [0.0], states, 0, **args)
    for k in range(3):
        grads = [torch.from_numpy(g * f32(0.5) ** k).cuda()]
        with np.errstate(all="ignore"):
            o.step(grads)
            plain.step(grads)
        w, m, v = (x.cpu().numpy() for x in o.values())
        assert np.array_equal(m, plain.m, equal_nan=True) and np.array_equal(v, plain.v, equal_nan=True)
        assert np.array_equal(np.isnan(w), np.isnan(plain.want))
        fine = np.isfinite(plain.want)
        assert (np.abs(w - plain.want) <= plain.tol)[fine].all()
        if states == "8bit":
            assert ((plain.vc > 0) | ~(plain.v > 0)).all()
        plain.w = w


def test_adamw_moments_in_8_bits_move_as_they_should(ev):
    """v with gradients of one: 1 - 0.999^t on average, though a step moves it by far less than a code's step.  65536 places:
    their codes are a tenth of v apart, and the mean of a walk of t steps is off by less than v sqrt(t 0.001 / 65536)."""
    n = 65536
    params = [torch.zeros(n, device="cuda")]
    o = ev.adamw(params, lr=0.0, states="8bit", seed=3)
    g = [torch.ones(n, device="cuda")]
    for t in range(1, 301):
        o.step(g)
        if t in (1, 10, 100, 300):
            m, v = (x.double() for x in o.values("mv"))
            want = 1 - 0.999 ** t
            # five times the deviation of the mean: each step rounds by at most half a code's step of 12.5 %, in its own way
            assert abs(float(v.mean()) / want - 1) < 5 * 0.0625 * math.sqrt(t / n)
            assert abs(float(m.mean()) / (1 - 0.9 ** t) - 1) < 5 * 0.0625 * math.sqrt(10 / n)


def test_adamw_of_bf16_parameters_loses_nothing(ev):
    """Steps a thousandth of a bf16 step: after 2000 of them the parameter has moved as an fp32 one has."""
    a, b = torch.full((300,), 1.0, device="cuda"), torch.full((300,), 1.0, dtype=torch.bfloat16, device="cuda")
    oa, ob = (ev.adamw([x], lr=2e-6, weight_decay=0.0) for x in (a, b))
    g = torch.ones(300, device="cuda")
    for _ in range(2000):
        oa.step([g])
        ob.step([g])
    assert torch.equal(oa.values("w")[0], ob.values("w")[0]) and torch.equal(ob.values("w")[0][:300], a)
    assert abs(float(b[0]) - float(a[0])) <= 2.0 ** -8 and float(a[0]) < 0.9961


def test_adamw_parameters_written_anew(ev):
    """A bf16 parameter that its owner sets, the low halves as they are: taken to within half a rounding, zero as (next to) zero."""
    p = torch.full((256,), 0.1, dtype=torch.bfloat16, device="cuda")
    o = ev.adamw([p], lr=1e-3, weight_decay=0.0)
    o.low[:256] = torch.arange(-32768, 32768, 256, dtype=torch.int32).to(torch.int16).cuda()
    new = torch.tensor([0.0, -0.0, 1.0, -1.0, 2.0 ** -126, 3.0e38, 0.5, -7.0], device="cuda").repeat(32)
    p.copy_(new)
    w = o.values("w")[0]
    assert torch.isfinite(w).all() and ((w - p.float()).abs() <= 2.0 ** -8 * p.float().abs() + 2.0 ** -133).all()
    o.low.zero_()
    assert torch.equal(o.values("w")[0], p.float())


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_adamw_state_is_what_is_saved(ev, states):
    """A second optimiser that takes over parameters and state goes on bit for bit."""
    params = tensors_of(LISTS["ragged"], "mixed")
    o = ev.adamw(params, states=states, seed=9)
    for k in range(2):
        o.step(grads_of(params, k))
    other = [p.clone() for p in params]
    q = ev.adamw(other, states=states, seed=9)
    for name in ("m", "v", "m_exponent", "v_exponent", "low", "steps"):
        if getattr(o, name) is not None:
            getattr(q, name).copy_(getattr(o, name))
    for k in range(2, 4):
        o.step(grads_of(params, k))
        q.step(grads_of(params, k))
    assert all(torch.equal(a, b) for a, b in zip(params, other)) and all(torch.equal(a, b) for a, b in zip(o.values(), q.values()))


# ---------------------------------------------------------------------------
# together, as they are used
# ---------------------------------------------------------------------------
class Loop:
    """A training step of kinds -> norm -> dense layer -> squared error, on operators only; the state of a second one to check
    it by."""

    def __init__(self, ev, dtype, states, rows=3001, kinds=37, C=96, N=40):
        t = TYPES[dtype]
        self.ev, self.kinds, self.C, self.rows = ev, kinds, C, rows
        self.params = [rand(1, kinds, C).to(t).cuda(), (1 + 0.1 * rand(2, C)).float().cuda(), (0.1 * rand(3, C)).float().cuda(),
                       (rand(4, C, N) / math.sqrt(C)).to(t).cuda(), (0.1 * rand(5, N)).float().cuda()]
        self.ids, self.goal = ids_of(rows, kinds, "padding").cuda(), rand(6, rows, N).to(t).cuda()
        self.opt = ev.adamw(self.params, lr=1e-2, weight_decay=[0.01, 0, 0, 0.01, 0], states=states, seed=5)

    def gradients(self):
        ev, (table, gamma, beta, w, b) = self.ev, self.params
        x = ev.embed_rows(self.ids, table, 1.5)
        u, mean, rstd = ev.row_norm(x, gamma, beta, EPS, "silu")
        y = ev.dense(u, w, b)
        dy = (y - self.goal) * (1 / 1024)
        du, dw, db = ev.dense_backward(dy, u, w)
        dx, dgamma, dbeta = ev.row_norm_backward(du, x, gamma, beta, mean, rstd, "silu")
        return y, [ev.embed_rows_backward(dx, self.ids, self.kinds, 1.5), dgamma, dbeta, dw, db]

    def step(self):
        y, grads = self.gradients()
        self.opt.step(grads)
        return y, grads


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step(ev, dtype):
    """Its gradients against autograd in 64 bits on the values of each storage step: in norm within 4 roundings of the storage
    type for each of the four tensors on the way, 2^-18 for fp32."""
    loop = Loop(ev, dtype, "f32")
    t = TYPES[dtype]
    y, grads = loop.gradients()
    table, gamma, beta, w, b = (p.double().cpu().requires_grad_() for p in loop.params)
    ids = loop.ids.cpu().long()
    x = torch.where((ids >= 0)[:, None], table[ids.clamp(min=0)] * 1.5, torch.zeros((), dtype=torch.float64))
    c = x - x.mean(1, keepdim=True)
    u = act(gamma * c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) + beta, "silu")
    out = u @ w + b
    (out.detach() - loop.goal.double().cpu()).mul(1 / 1024)
    out.backward((out.detach() - loop.goal.double().cpu()) / 1024)
    most = 4 * 4 * R(t) if t == torch.bfloat16 else 2.0 ** -18
    for g, p, what in zip(grads, (table, gamma, beta, w, b), ("table", "gamma", "beta", "w", "b")):
        off = float((g.double().cpu() - p.grad).norm() / p.grad.norm())
        assert off <= most, (what, off)


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step_on_another_stream_and_in_a_graph(ev, dtype, states):
    """Steps of a loop on the current stream, of one on a stream of its own, and of two captured ones, replayed with eager work in
    between: the same bits, and a captured step counts on."""
    def bits(loop):
        return [p.clone() for p in loop.params] + list(loop.opt.values()) + [loop.opt.steps.clone()]
    eager, other = Loop(ev, dtype, states), Loop(ev, dtype, states)
    captured = [Loop(ev, dtype, states) for _ in range(2)]
    for loop in [eager, other] + captured:
        loop.step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = []
    for loop in captured:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = loop.step()
        graphs.append((g, out))
    for k in range(4):
        y, grads = eager.step()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other.step()
        for (g, out), loop in zip(graphs, captured):
            g.replay()
        torch.cuda.synchronize()
        want = bits(eager)
        assert int(want[-1][0]) == k + 2
        for loop in [other] + captured:
            assert all(torch.equal(a, b) for a, b in zip(bits(loop), want)), k
        for _, out in graphs:
            assert torch.equal(out[0], y) and all(torch.equal(a, b) for a, b in zip(out[1], grads)), k
        torch.cuda.synchronize()


def test_calls_on_two_streams_at_once(ev):
    """Large calls of one context side by side, workspaces of their own: the bits of calls one after the other."""
    rows, C, kinds = 60011, 128, 300
    x, dy, ids = rand(1, rows, C).float().cuda(), rand(2, rows, C).float().cuda(), ids_of(rows, kinds, "skewed").cuda()

    def work():
        y, mean, rstd = ev.row_norm(x)
        return (y, ev.embed_rows_backward(dy, ids, kinds)) + ev.row_norm_backward(dy, x, None, None, mean, rstd)
    want = work()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(work())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


@pytest.mark.parametrize("dtype,C", [("bf16", 64), ("f32", 128), ("bf16", 256), ("f32", 256), ("bf16", 512), ("f32", 512), ("bf16", 1024), ("f32", 1024), ("f32", 8192),
                                     ("bf16", 16384), ("f32", 16384)])
def test_row_norm_of_more_than_the_caches(ev, dtype, C):
    """Rows of together more than 256 MiB: each the same as among few, and gamma's and beta's gradients by 64 bits."""
    t = TYPES[dtype]
    rows = 2 ** 28 // (C * (2 if dtype == "bf16" else 4)) + 5
    g = torch.Generator(device="cuda").manual_seed(C)
    x, dy = torch.randn(rows, C, generator=g, device="cuda").to(t), torch.randn(rows, C, generator=g, device="cuda").to(t)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device="cuda"), 0.3 * torch.randn(C, generator=g, device="cuda")
    y, mean, rstd = ev.row_norm(x, gamma, beta, EPS, "silu")
    step = rows // 3
    for rest, past in ((x, dy), (ev.keep_rows(x), None)):
        dx, dgamma, dbeta = ev.row_norm_backward(dy, rest, gamma, beta, mean, rstd, "silu", past)
        back = x if rest is x else ev.restore_rows(rest, torch.float32)
        sums = torch.zeros(4, C, dtype=torch.float64, device="cuda")
        for lo in range(0, rows, step):
            at = slice(lo, min(lo + step, rows))
            few = ev.row_norm(x[at], gamma, beta, EPS, "silu")
            assert torch.equal(few[0], y[at]) and torch.equal(few[1], mean[at]) and torch.equal(few[2], rstd[at])
            # codes go by rows, so those of a part are the part's own
            part = x[at] if rest is x else ev.keep_rows(x[at])
            assert torch.equal(ev.row_norm_backward(dy[at], part, gamma, beta, mean[at], rstd[at], "silu", None if past is None else past[at])[0], dx[at])
            for lo2 in range(at.start, at.stop, 1 << 24 >> (C.bit_length() - 1)):
                to = slice(lo2, min(lo2 + (1 << 24 >> (C.bit_length() - 1)), at.stop))
                xh = (back[to].double() - mean[to, None]) * rstd[to, None]
                dz = dy[to].double() * slope(xh * gamma + beta, "silu")
                sums += torch.stack([(dz * xh).sum(0), dz.sum(0), (dz * xh).abs().sum(0), dz.abs().sum(0)])
        # 64 rows of a thread, its runs (of at most 256 workgroups' rows a run, here fewer than 70), 64 bits twice; the terms' own 30
        n = 64 + 70 + 6 + 30
        size = 1 + gamma.abs().double() + beta.abs()
        close(dgamma, sums[0].cpu(), (n * U * (sums[2] + sums[3] * size)).cpu(), "dgamma")
        close(dbeta, sums[1].cpu(), (n * U * sums[3] * size).cpu(), "dbeta")


def test_offsets_beyond_32_bits(ev):
    """Arrays of more than 4 GiB: the last rows against 64 bits, everything that is summed over all rows too."""
    rows, C, per, kinds = 8_600_000, 128, 500, 1000
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(rows, C, generator=g, device="cuda")
    one = torch.ones(C), torch.zeros(C)
    last = slice(rows - per, rows)
    tail = x[last].cpu()
    y, mean, rstd = ev.row_norm(x, eps=EPS, act="silu")
    check_norm(tail, *one, "silu", torch.float32, (y[last], mean[last], rstd[last]))
    dx, dgamma, dbeta = ev.row_norm_backward(x, x, None, None, mean, rstd, "silu", out=y)
    ref = norm_back_reference(tail, tail, None, *one, mean[last].cpu(), rstd[last].cpu(), "silu", torch.float32)
    close(dx[last], *ref[0], "dx")
    sums = torch.zeros(4, C, dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 1_000_000):
        v = x[lo:lo + 1_000_000].double()
        xh = (v - mean[lo:lo + 1_000_000, None]) * rstd[lo:lo + 1_000_000, None]
        dz = v * slope(xh, "silu")
        sums += torch.stack([(dz * xh).sum(0), dz.sum(0), (dz * xh).abs().sum(0), dz.abs().sum(0)])
    # 64 rows of a thread, its runs (128 rows of a workgroup's 16 or more at a time on 256 CUs), 64 bits twice; the terms' own 30
    n = 64 + rows / (256 * 16 * 64) + 6 + 30
    close(dgamma, sums[0].cpu(), (n * U * sums[2]).cpu(), "dgamma")
    close(dbeta, sums[1].cpu(), (n * U * sums[3]).cpu(), "dbeta")
    # rows by kind, and a table of as many kinds
    ids = torch.randint(0, kinds, (rows,), generator=g, device="cuda", dtype=torch.int32)
    ev.embed_rows(ids, x[:kinds], 2.0, out=y)
    assert torch.equal(y[last], x[ids[last].long()] * 2)
    far = torch.tensor([rows - 1, 3, rows - 77], dtype=torch.int32, device="cuda")
    assert torch.equal(ev.embed_rows(far, x), x[far.long()])
    dt = ev.embed_rows_backward(x, ids, kinds)
    want, size = (torch.zeros(kinds, C, dtype=torch.float64, device="cuda") for _ in range(2))
    for lo in range(0, rows, 1_000_000):
        v = x[lo:lo + 1_000_000].double()
        want.index_add_(0, ids[lo:lo + 1_000_000].long(), v)
        size.index_add_(0, ids[lo:lo + 1_000_000].long(), v.abs())
    # 64 rows of a run and four runs of a chunk in fp32, five lists rounded to fp32
    close(dt, want.cpu(), ((64 + 4 + 5) * U * size + 2 * U * want.abs()).cpu(), "dtable")
    y.fill_(7)
    ev.embed_rows_backward(x[:3], far, rows, out=y)
    assert torch.equal(y[far.long()], x[:3]) and not y[last][:per - 77].any() and int((y != 0).any(1).sum()) == 3


@pytest.mark.parametrize("rows", [1, 4096, 4097, 70001])
def test_the_most_kinds(ev, rows):
    """Kinds up to the largest number of them, of which most have no row."""
    kinds, C = 2 ** 31 - 1, 1
    g = torch.Generator().manual_seed(rows)
    ids = torch.randint(0, kinds, (rows,), generator=g)
    ids[0], ids[rows // 2], ids[-1] = kinds - 1, 0, kinds - 1
    if rows > 1:
        ids[1] = -1
    dy = rand(3, rows, C).bfloat16()
    dt = ev.embed_rows_backward(dy.cuda(), ids.int().cuda(), kinds)
    used, back = ids[ids >= 0].unique(return_inverse=True)
    want, size = (torch.zeros(used.numel(), C, dtype=torch.float64).index_add_(0, back, v[ids >= 0]) for v in (dy.double(), dy.double().abs()))
    close(dt[used.cuda()], want, 4 * U * size + (R(torch.bfloat16) + 3 * U) * want.abs(), "dtable")
    assert sum(int(part.count_nonzero()) for part in dt.split(2 ** 29)) == int((want != 0).sum())
    y = ev.embed_rows(ids.int().cuda(), dt, 2.0)
    assert torch.equal(y, torch.where(ids.cuda()[:, None] >= 0, 2 * dt[ids.cuda().clamp(min=0)], 0))
    assert ev.check() == 0


@pytest.mark.parametrize("states,n", [("f32", 2 ** 30 + 131 * 128 + 5), ("8bit", 2 ** 31 + 131 * 128 + 5)])
def test_adamw_beyond_32_bits(ev, states, n):
    """One tensor of more than 4 GiB (and more than 2^31 places): its last elements."""
    t = torch.float32 if states == "f32" else torch.bfloat16
    p, g = torch.zeros(n, dtype=t, device="cuda"), torch.zeros(n, dtype=t, device="cuda")
    first = (n - 3000) // 128 * 128
    p[first:].copy_(0.1 * rand(1, n - first))
    g[first:].copy_(rand(2, n - first))
    args = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8)
    o, plain = ev.adamw([p], **args, weight_decay=0.1, states=states, seed=4), Plain([p[first:]], [0.1], states, 4, **args)
    plain.first = first
    o.step([g])
    plain.step([g[first:]])
    if states == "f32":
        off = np.abs(p[first:].double().cpu().numpy() - plain.want[:n - first])
        assert (off <= plain.tol[:n - first]).all()
        assert np.array_equal(o.m[first:].cpu().numpy(), plain.m) and np.array_equal(o.v[first:].cpu().numpy(), plain.v)
        assert not p[:first].any() and not o.m[:first].any()
    else:
        assert np.array_equal(o.m[first:].cpu().numpy(), plain.mc) and np.array_equal(o.v[first:].cpu().numpy(), plain.vc)
        assert np.array_equal(o.m_exponent[first // 128:].cpu().numpy(), plain.me) and np.array_equal(o.v_exponent[first // 128:].cpu().numpy(), plain.ve)
        off = np.abs(p[first:].double().cpu().numpy() - plain.want[:n - first])
        assert (off <= plain.tol[:n - first] + 2.0 ** -8 * np.abs(plain.want[:n - first])).all()
        assert not p[:first].any() and not o.m[:first].any() and not o.low[:first].any()
    assert o.steps.tolist() == [1, 0]


# ---------------------------------------------------------------------------
# workspaces and refusals
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", [(1, 1), (3, 8192), (66559, 32), (5003, 520), (1201, 16384), (65617, 175)])
def test_row_norm_stays_in_its_workspace(B, ev, dtype, rows, C):
    t = TYPES[dtype]
    x, dy = rand(1, rows, C).to(t).cuda(), rand(2, rows, C).to(t).cuda()
    dx, stats, vec = torch.empty_like(x), torch.ones(2, rows, device="cuda"), torch.empty(2, C, device="cuda")
    size = B.dc_row_norm_bytes(ev.ctx, rows, C)
    buf = torch.full((size + (4 << 20),), 77, dtype=torch.uint8, device="cuda")
    ws = buf[2 << 20:(2 << 20) + size]
    torch.cuda.synchronize()
    args = B.DcRowNormArgs(dtype=B.DC_BF16 if dtype == "bf16" else B.DC_F32, act=3, rows=rows, channels=C, X=x.data_ptr(), ldx=C, mean=stats[0].data_ptr(),
                           rstd=stats[1].data_ptr(), dY=dy.data_ptr(), lddy=C, dX=dx.data_ptr(), lddx=C, dgamma=vec[0].data_ptr(), dbeta=vec[1].data_ptr(),
                           workspace=ws.data_ptr(), workspace_bytes=size)
    assert B.dc_row_norm_backward(ev.ctx, args) == B.DC_OK
    torch.cuda.synchronize()
    assert (buf[:2 << 20] == 77).all() and (buf[(2 << 20) + size:] == 77).all()
    args.workspace_bytes = size - 1
    assert B.dc_row_norm_backward(ev.ctx, args) == B.DC_ERR_CAPACITY
    # without the vectors no workspace is taken
    args.dgamma = args.dbeta = args.workspace = None
    got = dx.clone()
    dx.zero_()
    torch.cuda.synchronize()
    assert B.dc_row_norm_backward(ev.ctx, args) == B.DC_OK
    torch.cuda.synchronize()
    assert torch.equal(dx, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,kinds,C", [(1, 1, 1), (17, 3, 8), (4096, 511, 40), (4097, 512, 33), (70001, 300000, 5), (300007, 2, 4), (0, 9, 9)])
def test_embed_rows_stays_in_its_workspace(B, ev, dtype, rows, kinds, C):
    t = TYPES[dtype]
    dy, ids, dt = rand(2, rows, C).to(t).cuda(), ids_of(rows, kinds, "skewed").cuda(), torch.empty(kinds, C, dtype=t, device="cuda")
    size = B.dc_embed_rows_bytes(ev.ctx, rows, kinds, C)
    buf = torch.full((size + (4 << 20),), 77, dtype=torch.uint8, device="cuda")
    ws = buf[2 << 20:(2 << 20) + size]
    torch.cuda.synchronize()
    args = B.DcEmbedRowsArgs(dtype=B.DC_BF16 if dtype == "bf16" else B.DC_F32, rows=rows, kinds=kinds, channels=C, scale=1.0, id=ids.data_ptr(), dY=dy.data_ptr(),
                             lddy=C, dtable=dt.data_ptr(), ld_dtable=C, workspace=ws.data_ptr(), workspace_bytes=size)
    assert B.dc_embed_rows_backward(ev.ctx, args) == B.DC_OK
    torch.cuda.synchronize()
    assert (buf[:2 << 20] == 77).all() and (buf[(2 << 20) + size:] == 77).all()
    args.workspace_bytes = size - 1
    if size:
        assert B.dc_embed_rows_backward(ev.ctx, args) == B.DC_ERR_CAPACITY


def test_row_norm_refuses(B, ev):
    x, y, s = (torch.zeros(4, 8, device="cuda") for _ in range(3))
    ok = dict(dtype=B.DC_F32, act=0, rows=4, channels=8, eps=1e-5, X=x.data_ptr(), ldx=8, mean=s[0].data_ptr(), rstd=s[1].data_ptr(), Y=y.data_ptr(), ldy=8)
    assert B.dc_row_norm(ev.ctx, B.DcRowNormArgs(**ok)) == B.DC_OK
    for bad, want in [(dict(dtype=2), 1), (dict(act=4), 1), (dict(rows=-1), 1), (dict(rows=1 << 31), 7), (dict(channels=0), 1), (dict(channels=16385), 7),
                      (dict(eps=0.0), 1), (dict(eps=math.nan), 1), (dict(X=0), 1), (dict(Y=0), 1), (dict(ldx=7), 1), (dict(ldy=1 << 23), 7), (dict(mean=0), 1),
                      (dict(X=x.data_ptr() + 2), 1), (dict(gamma=s.data_ptr() + 1), 1), (dict(Y=x.data_ptr() + 16), 1), (dict(Y=s.data_ptr()), 1),
                      (dict(mean=x.data_ptr()), 1), (dict(rstd=s[0].data_ptr() + 4), 1)]:
        assert B.dc_row_norm(ev.ctx, B.DcRowNormArgs(**{**ok, **bad})) == want, bad
        assert B.dc_last_error(ev.ctx)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    back = dict(dtype=B.DC_F32, act=0, rows=4, channels=8, X=x.data_ptr(), ldx=8, mean=s[0].data_ptr(), rstd=s[1].data_ptr(), dY=y.data_ptr(), lddy=8,
                dX=y.data_ptr(), lddx=8, dgamma=s[2].data_ptr(), dbeta=s[3].data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    assert B.dc_row_norm_backward(ev.ctx, B.DcRowNormArgs(**back)) == B.DC_OK
    for bad, want in [(dict(mean=0), 1), (dict(dY=0), 1), (dict(dX=0), 1), (dict(dbeta=0), 1), (dict(workspace=0), 4), (dict(workspace_bytes=8), 4),
                      (dict(workspace=ws.data_ptr() + 4), 1), (dict(dX=y.data_ptr() + 4), 1), (dict(dX=s.data_ptr()), 1), (dict(dres=y.data_ptr(), lddres=9), 1),
                      (dict(dbeta=s[2].data_ptr() + 4), 1), (dict(workspace=y.data_ptr()), 1)]:
        assert B.dc_row_norm_backward(ev.ctx, B.DcRowNormArgs(**{**back, **bad})) == want, bad
    torch.cuda.synchronize()
    assert ev.check() == B.DC_OK


def test_embed_rows_refuses(B, ev):
    x, y, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ok = dict(dtype=B.DC_F32, rows=4, kinds=4, channels=8, scale=1.0, id=ids.data_ptr(), table=x.data_ptr(), ld_table=8, Y=y.data_ptr(), ldy=8)
    assert B.dc_embed_rows(ev.ctx, B.DcEmbedRowsArgs(**ok)) == B.DC_OK
    for bad, want in [(dict(dtype=-1), 1), (dict(rows=-1), 1), (dict(rows=1 << 31), 7), (dict(kinds=0), 1), (dict(channels=0), 1), (dict(channels=65537), 7),
                      (dict(id=0), 1), (dict(id=ids.data_ptr() + 2), 1), (dict(table=0), 1), (dict(ld_table=7), 1), (dict(Y=0), 1), (dict(ldy=7), 1),
                      (dict(Y=x.data_ptr()), 1), (dict(Y=ids.data_ptr(), rows=1), 1)]:
        assert B.dc_embed_rows(ev.ctx, B.DcEmbedRowsArgs(**{**ok, **bad})) == want, bad
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    back = dict(dtype=B.DC_F32, rows=4, kinds=4, channels=8, scale=1.0, id=ids.data_ptr(), dY=x.data_ptr(), lddy=8, dtable=y.data_ptr(), ld_dtable=8,
                workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    assert B.dc_embed_rows_backward(ev.ctx, B.DcEmbedRowsArgs(**back)) == B.DC_OK
    for bad, want in [(dict(dY=0), 1), (dict(dtable=0), 1), (dict(ld_dtable=4), 1), (dict(workspace=0), 4), (dict(workspace_bytes=8), 4),
                      (dict(workspace=ws.data_ptr() + 8), 1), (dict(dtable=x.data_ptr()), 1), (dict(workspace=x.data_ptr()), 1)]:
        assert B.dc_embed_rows_backward(ev.ctx, B.DcEmbedRowsArgs(**{**back, **bad})) == want, bad
    torch.cuda.synchronize()
    assert ev.check() == B.DC_OK


def test_adamw_refuses(B, ev):
    p, g, m, v = (torch.zeros(256, device="cuda") for _ in range(4))
    low, steps, e = torch.zeros(256, dtype=torch.int16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.uint8, device="cuda")

    def call(listed=(), fn=None, **more):
        one = dict(p=p.data_ptr(), g=g.data_ptr(), n=200, at=0, p_dtype=0, g_dtype=0, weight_decay=0.0)
        table = (B.DcAdamwTensor * max(1, len(listed)))(*[B.DcAdamwTensor(**{**one, **t}) for t in listed])
        args = dict(moments=0, n_tensors=len(listed), tensors=B.C.addressof(table), total=256, m=m.data_ptr(), v=v.data_ptr(), low=low.data_ptr(),
                    steps=steps.data_ptr(), lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8)
        return (fn or B.dc_adamw)(ev.ctx, B.DcAdamwArgs(**{**args, **more}))
    assert call([{}]) == B.DC_OK and call([]) == B.DC_OK
    for bad in [dict(n=-1), dict(at=64), dict(at=-128), dict(n=257), dict(at=128, n=129), dict(p=0), dict(p=p.data_ptr() + 2), dict(g=g.data_ptr() + 1), dict(p_dtype=2),
                dict(g_dtype=-1), dict(weight_decay=-1.0), dict(weight_decay=math.nan), dict(p=g.data_ptr()), dict(p=m.data_ptr()), dict(p=steps.data_ptr(), n=1),
                dict(g=v.data_ptr())]:
        assert call([bad]) == B.DC_ERR_INVALID_ARG, bad
        assert B.dc_last_error(ev.ctx)
    # the same tensor twice, places that are not behind the last one's
    assert call([dict(n=128), dict(n=128, at=128)]) == B.DC_ERR_INVALID_ARG
    assert call([dict(n=100), dict(n=100, at=128, p=p.data_ptr() + 400)]) == B.DC_OK       # a shared gradient is none of them
    assert call([dict(n=129), dict(n=10, at=128, p=p.data_ptr() + 800)]) == B.DC_ERR_INVALID_ARG
    for bad, want in [(dict(moments=2), 1), (dict(n_tensors=-1), 1), (dict(tensors=0), 1), (dict(total=200), 1), (dict(total=-128), 1), (dict(total=1 << 39), 7), (dict(m=0), 1),
                      (dict(v=v.data_ptr() + 4), 1), (dict(moments=1), 1), (dict(steps=0), 1), (dict(steps=steps.data_ptr() + 2), 1), (dict(grad_scale=g.data_ptr() + 2), 1),
                      (dict(lr=-1.0), 1), (dict(lr=math.nan), 1), (dict(beta1=1.0), 1), (dict(beta2=-0.1), 1), (dict(eps=0.0), 1), (dict(eps=1e-60), 1), (dict(v=m.data_ptr()), 1),
                      (dict(grad_scale=m.data_ptr()), 1), (dict(moments=1, m_exponent=e.data_ptr(), v_exponent=e.data_ptr() + 1), 1)]:
        assert call([{}], **bad) == want, bad
    assert call([dict(p_dtype=1)], low=0) == B.DC_ERR_INVALID_ARG
    out = torch.zeros(256, device="cuda")
    values = lambda w: lambda ctx, a: B.dc_adamw_values(ctx, a, w, 0, 0)   # noqa: E731
    assert call([dict(g=0)], values(out.data_ptr()), lr=-1.0, steps=0) == B.DC_OK
    for w in (out.data_ptr() + 4, p.data_ptr(), m.data_ptr()):
        assert call([{}], values(w)) == B.DC_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert ev.check() == B.DC_OK and not p.any() and steps.tolist() == [3, 0]


def test_embed_rows_says_what_was_wrong_with_an_id(B, ev):
    assert ev.check() == B.DC_OK
    ev.embed_rows(torch.tensor([0, 9], dtype=torch.int32, device="cuda"), torch.ones(9, 8, device="cuda"))
    assert ev.check() == B.DC_ERR_INVALID_ARG and "id outside [-1, kinds)" in B.dc_last_error(ev.ctx)
    assert ev.check() == B.DC_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("C", [40, 256, 600, 9001])
@pytest.mark.parametrize("where", ["x", "dy", "residual"])
def test_row_norm_backward_of_a_row_that_is_not_finite(ev, dtype, bad, C, where):
    """The other rows have the bits that they have where that row is finite."""
    x, gamma, beta = (v.cuda() for v in norm_inputs(50, C, dtype))
    t = {"x": x, "dy": rand(9, 50, C).to(x.dtype).cuda(), "residual": rand(10, 50, C).to(x.dtype).cuda()}

    def back():
        _, mean, rstd = ev.row_norm(t["x"], gamma, beta, EPS, "silu")
        return ev.row_norm_backward(t["dy"], t["x"], gamma, beta, mean, rstd, "silu", t["residual"])
    clean = back()
    t[where][7, C // 2] = bad
    dx, dgamma, dbeta = back()
    fine = torch.arange(50, device="cuda") != 7
    assert torch.equal(dx[fine], clean[0][fine]) and not torch.isfinite(dx[7, C // 2])
    if where == "residual":                                # which is added behind everything else
        assert torch.equal(dgamma, clean[1]) and torch.equal(dbeta, clean[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,spread", [(1e5, 1.0), (1e6, 0.1), (-1e8, 8.0), (0.0, 1e-6), (3e12, 1e9)])
@pytest.mark.parametrize("C", [5, 200, 3000, 9001])
@pytest.mark.parametrize("name", ["none", "silu"])
def test_row_norm_backward_far_from_zero(ev, dtype, offset, spread, C, name):
    """Gradients by the mean and rstd that are given: those of the forward pass, which are rounded."""
    rows, t = 40, TYPES[dtype]
    x, dy = (offset + spread * rand(3, rows, C)).to(t), rand(4, rows, C).to(t)
    _, gamma, beta = norm_inputs(1, C, dtype)
    _, mean, rstd = ev.row_norm(x.cuda(), gamma.cuda(), beta.cuda(), EPS, name)
    got = ev.row_norm_backward(dy.cuda(), x.cuda(), gamma.cuda(), beta.cuda(), mean, rstd, name)
    for g, (w, tol), what in zip(got, norm_back_reference(x, dy, None, gamma, beta, mean.cpu(), rstd.cpu(), name, t), ("dx", "dgamma", "dbeta")):
        close(g, w, tol, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,ld,first", [(64, 65, 1), (128, 131, 3), (256, 257, 1), (256, 259, 2), (512, 513, 7), (1024, 1025, 1), (4096, 4099, 1), (8192, 8195, 5), (16384, 16387, 1)])
def test_row_norm_of_more_than_the_caches_anywhere(ev, dtype, C, ld, first):
    """Rows of together more than 256 MiB that begin at any element have the bits of rows on 16-byte boundaries, both ways, from
    kept rows and in place, and nothing between them is touched."""
    t = TYPES[dtype]
    rows = 2 ** 28 // (C * (2 if dtype == "bf16" else 4)) + 5
    g = torch.Generator(device="cuda").manual_seed(C + ld)

    def spread_out(v, fill, cols=C):
        apart = ld - C + cols
        buf = torch.full((first + v.shape[0] * apart,), fill, dtype=v.dtype, device="cuda")
        w = buf[first:].view(v.shape[0], apart)[:, :cols]
        w.copy_(v)
        return w, buf

    def untouched(w, buf, fill):
        w.fill_(fill)
        return bool((buf == fill).all())
    x, dy, past = (torch.randn(rows, C, generator=g, device="cuda").to(t) for _ in range(3))
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device="cuda"), 0.3 * torch.randn(C, generator=g, device="cuda")
    want = ev.row_norm(x, gamma, beta, EPS, "silu")
    xa, _ = spread_out(x, 3)
    ya, buf = spread_out(x, 5)
    got = ev.row_norm(xa, gamma, beta, EPS, "silu", out=ya)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and untouched(ya, buf, 5)
    del ya, buf, got
    mean, rstd = want[1:]
    want = ev.row_norm_backward(dy, x, gamma, beta, mean, rstd, "silu", past)
    da, _ = spread_out(dy, 3)
    pa, buf = spread_out(past, 5)
    got = ev.row_norm_backward(da, xa, gamma, beta, mean, rstd, "silu", pa, out=pa)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and untouched(pa, buf, 5)
    del pa, buf, got, xa
    kept = ev.keep_rows(x)
    want = ev.row_norm_backward(dy, kept, gamma, beta, mean, rstd, "silu")
    off = type(kept)(spread_out(kept.code, 3)[0], spread_out(kept.exponent, 3, C // 32)[0], C)
    ya, buf = spread_out(x, 5)
    got = ev.row_norm_backward(da, off, gamma, beta, mean, rstd, "silu", out=ya)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and untouched(ya, buf, 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kinds,how", [(97, "skewed"), (20011, "even")])
@pytest.mark.parametrize("C,ld,first", [(1031, 1033, 1), (2057, 2058, 3), (264, 265, 1), (520, 520, 1)])
def test_embed_rows_backward_of_more_than_the_caches_anywhere(ev, dtype, kinds, how, C, ld, first):
    """Rows of together more than 256 MiB that begin at any element, to a table that does: against sums in 64 bits, and the bits
    of rows one behind the other."""
    t = TYPES[dtype]
    rows = 2 ** 28 // (C * (2 if dtype == "bf16" else 4)) + 5
    print(rows, kinds, C, ld, first, flush=True)
    dy = torch.randn(rows, C, generator=torch.Generator(device="cuda").manual_seed(C + ld), device="cuda").to(t)
    ids = ids_of(rows, kinds, how).cuda()
    da = torch.full((first + rows * ld,), math.nan, dtype=t, device="cuda")[first:].view(rows, ld)[:, :C]
    da.copy_(dy)
    buf = torch.full((first + kinds * ld,), 5, dtype=t, device="cuda")
    table = buf[first:].view(kinds, ld)[:, :C]
    ev.embed_rows_backward(da, ids, kinds, 0.7, out=table)
    assert torch.equal(table, ev.embed_rows_backward(dy, ids, kinds, 0.7))
    want, size = (torch.zeros(kinds, C, dtype=torch.float64, device="cuda") for _ in range(2))
    for lo in range(0, rows, 30000):
        v = dy[lo:lo + 30000].double()
        want.index_add_(0, ids[lo:lo + 30000].long(), v)
        size.index_add_(0, ids[lo:lo + 30000].long(), v.abs())
    # 64 rows of a run and four runs of a chunk in fp32, three lists rounded to fp32, the scale as fp32 and its product
    close(table, (0.7 * want).cpu(), ((64 + 4 + 3) * U * 0.7 * size + (R(t) + 3 * U) * 0.7 * want.abs()).cpu(), "dtable")
    table.fill_(5)
    assert (buf == 5).all()
