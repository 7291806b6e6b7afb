"""The operators on rows of a batch (dense layer with epilogue, norm over the rows of each graph, rows kept in 8 bits, and
their gradients) against plain implementations in 64 bits, element by element.

Tolerances count roundings.  U = 2^-24 is the most that rounding to fp32 is off by, relative to the value; R(t) =
finfo(t).eps / 2 the same for the storage type of an output.  A sum of products through the matrix cores rounds its
accumulator once per instruction and drops what lies below the accumulator's 24 bits, together at most 3 U of the
sum of the terms' sizes per instruction.
"""
import itertools
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
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


def product_roundings(K, t):
    """3 U per instruction: bf16 one per 16 indices; fp32 in pieces 24 per section of 64, one rounding per section and 2
    for the products that are left out."""
    return 3 * (K // 16 + 1) + 2 if t == torch.bfloat16 else 3 * 24 + K // 64 + 3


# ---------------------------------------------------------------------------
# dense
# ---------------------------------------------------------------------------
SHAPES = [(1, 1, 1), (1, 256, 256), (3, 5, 7), (17, 384, 128), (127, 129, 131), (128, 64, 128), (300, 768, 256), (1000, 201, 139),
          (257, 16, 512), (2, 2, 300), (515, 40, 24), (64, 1031, 8)]


def dense_reference(x, w, b, r, name, t):
    z = x.double() @ w.double()
    size = x.double().abs() @ w.double().abs()
    if b is not None:
        z, size = z + b.double(), size + b.double().abs()
    dz = (product_roundings(x.shape[1], t) + 2) * U * size
    y = act(z, name)
    # slopes of the activations are below 1.13; their evaluation: eight roundings of the size of z
    dy = 1.13 * dz + 8 * U * z.abs()
    if r is not None:
        y = y + r.double()
        dy = dy + U * y.abs()
    return z, dz + (R(t) + U) * z.abs(), y, dy + (R(t) + U) * y.abs()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
def test_dense(ev, dtype, shape, name):
    t, (rows, K, N) = TYPES[dtype], shape
    print(dtype, shape, name, flush=True)
    x, w = rand(1, rows, K).to(t), (rand(2, K, N) / math.sqrt(K)).to(t)
    b, r = rand(3, N).float(), rand(4, rows, N).to(t)
    z, tz, y, ty = dense_reference(x, w, b, r, name, t)
    got, pre = ev.dense(x.cuda(), w.cuda(), b.cuda(), name, r.cuda(), want_pre=True)
    close(pre, z, tz, "z")
    close(got, y, ty, "y")
    # without bias and residual
    _, _, y, ty = dense_reference(x, w, None, None, name, t)
    close(ev.dense(x.cuda(), w.cuda(), act=name), y, ty, "plain")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,first", [(0, 1), (3, 0), (8, 8), (1, 5)])
@pytest.mark.parametrize("shape", [(130, 64, 128), (33, 72, 40)])
def test_dense_rows_anywhere(ev, dtype, ld, first, shape):
    """Rows apart and off every boundary, the result in place of the residual; what lies between rows is not touched."""
    t, (rows, K, N) = TYPES[dtype], shape
    x, w, b, r = rand(1, rows, K).to(t), (rand(2, K, N) / math.sqrt(K)).to(t), rand(3, N).float(), rand(4, rows, N).to(t)
    _, _, y, ty = dense_reference(x, w, b, r, "silu", t)
    rv = off_grid(r, N + ld, first)
    got = ev.dense(off_grid(x, K + ld, first), off_grid(w, N + ld, first), b.cuda(), "silu", residual=rv, out=rv)
    close(got, y, ty, "y")
    buf = rv._base if rv._base is not None else rv
    assert int(torch.isnan(buf.flatten()).sum()) == first + rows * ld


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense_without_rows(ev, dtype):
    t = TYPES[dtype]
    x, w = torch.empty(0, 32, dtype=t, device="cuda"), torch.ones(32, 16, dtype=t, device="cuda")
    assert ev.dense(x, w).shape == (0, 16)
    dx, dw, db = ev.dense_backward(torch.empty(0, 16, dtype=t, device="cuda"), x, w)
    assert dx.shape == (0, 32) and not dw.any() and not db.any()


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, 3.4e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense_keeps_rows_apart(ev, dtype, value):
    """A number that is not finite, or as large as fp32 goes, changes its own row only, and there as arithmetic says."""
    t, rows, K, N = TYPES[dtype], 200, 96, 64
    x, w = rand(1, rows, K).to(t), (rand(2, K, N) / math.sqrt(K)).to(t)
    w[5] = w[5].abs() * 0.25 + 0.01
    clean = ev.dense(x.cuda(), w.cuda())
    x[7, 5] = value
    got = ev.dense(x.cuda(), w.cuda())
    others = torch.arange(rows) != 7
    assert torch.equal(got[others.cuda()], clean[others.cuda()])
    want = (x[7].double() @ w.double()).to(t)
    if value == 3.4e38:
        assert torch.allclose(got[7].cpu().double(), want.double(), rtol=1e-2 if dtype == "bf16" else 1e-6)
    else:
        assert torch.equal(torch.isnan(got[7]).cpu(), torch.isnan(want)) and (math.isnan(value) or torch.equal(got[7].cpu(), want))


# More than four 32 x 32 tiles per CU (256 of them): widths that end in every place of a tile, a wave's 64 columns and a vector,
# contractions of one to many steps, the smallest widths that tiles take.
TILED = [(33001, 32, 24), (9001, 201, 139), (4501, 70, 255), (7003, 129, 131), (3001, 1031, 390), (2203, 8, 513), (40001, 8, 4),
         (17003, 40, 65), (9007, 33, 129), (8200, 72, 256), (4100, 9, 260), (33000, 8, 5), (5000, 256, 257)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", TILED)
def test_dense_of_many_rows(ev, dtype, shape):
    test_dense(ev, dtype, shape, ["silu", "none", "relu", "gelu"][(shape[0] + shape[2]) % 4])


# Four of the largest tiles per CU, and between one and two of the next.
@pytest.mark.parametrize("dtype,shape", [("f32", (131200, 17, 139)), ("f32", (131100, 40, 130)), ("bf16", (262500, 9, 139)), ("bf16", (262300, 70, 130)),
                                         ("f32", (33100, 40, 70)), ("f32", (17000, 33, 129)), ("bf16", (132000, 40, 70)), ("bf16", (70000, 70, 129))])
def test_dense_of_the_most_rows(B, ev, dtype, shape):
    rows, K, N = shape
    test_dense(ev, dtype, shape, "silu" if K % 2 else "relu")
    test_dense_backward(B, ev, dtype, (rows, N, K), "relu", K % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,first", [(3, 1), (8, 8)])
@pytest.mark.parametrize("shape", [(9000, 72, 131), (4600, 33, 250)])
def test_dense_of_many_rows_anywhere(ev, dtype, ld, first, shape):
    test_dense_rows_anywhere(ev, dtype, ld, first, shape)


@pytest.mark.parametrize("value", [math.inf, math.nan, -3.4e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [64, 139])
def test_dense_of_many_rows_keeps_them_apart(ev, dtype, value, N):
    t, rows, K = TYPES[dtype], 20001, 96
    x, w = rand(1, rows, K).to(t), (rand(2, K, N) / math.sqrt(K)).to(t)
    w[5] = w[5].abs() * 0.25 + 0.01
    clean = ev.dense(x.cuda(), w.cuda())
    bad = [7, 12345, rows - 1]
    x[bad, 5] = value
    got = ev.dense(x.cuda(), w.cuda())
    others = torch.ones(rows, dtype=torch.bool)
    others[bad] = False
    assert torch.equal(got[others.cuda()], clean[others.cuda()])
    for i in bad:
        want = (x[i].double() @ w.double()).to(t)
        if abs(value) == 3.4e38:
            assert torch.allclose(got[i].cpu().double(), want.double(), rtol=1e-2 if dtype == "bf16" else 1e-6)
        else:
            assert torch.equal(torch.isnan(got[i]).cpu(), torch.isnan(want)) and (math.isnan(value) or torch.equal(got[i].cpu(), want))


def backward_reference(dy, x, w, z, name, t):
    """Gradients and their tolerances, all in 64 bits; x as the values that are multiplied."""
    d = dy.double()
    dz = d if name == "none" else d * slope(z.double(), name)
    # evaluating the slope: sixteen roundings of a quantity of size 1 + |z|; for bf16 dz is rounded once more
    edz = torch.zeros_like(d) if name == "none" else d.abs() * 16 * U * (1 + z.double().abs())
    operand = edz if t == torch.float32 or name == "none" else edz + R(t) * dz.abs()
    rows, N = dy.shape
    K = w.shape[0]
    aw, ax = w.double().abs(), x.double().abs()
    dx, dw, db = dz @ w.double().t(), x.double().t() @ dz, dz.sum(0)
    tx = operand @ aw.t() + product_roundings(N, t) * U * (dz.abs() @ aw.t()) + (R(t) + U) * dx.abs()
    # a section of a slab at a time, then the sections and the slabs in fp32 and 64 bits
    sections = 3 * 96 + rows // 64 + 4
    tw = ax.t() @ operand + sections * U * (ax.t() @ dz.abs()) + (R(t) + U) * dw.abs()
    tb = edz.sum(0) + 4 * U * dz.abs().sum(0)
    return (dx, tx), (dw, tw), (db, tb)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES + [(5000, 96, 32)])
@pytest.mark.parametrize("name,kept", [("none", False), ("relu", True), ("gelu", False), ("silu", True)])
def test_dense_backward(B, ev, dtype, shape, name, kept):
    t, (rows, K, N) = TYPES[dtype], shape
    print(dtype, shape, name, kept, flush=True)
    x, w, dy, z = rand(1, rows, K).to(t), (rand(2, K, N) / math.sqrt(K)).to(t), rand(3, rows, N).to(t), rand(4, rows, N).to(t)
    xd = x.cuda()
    if kept:
        xd = ev.keep_rows(xd)
        x = ev.restore_rows(xd, torch.float32).cpu()
    ref = backward_reference(dy, x, w, z, name, t)
    got = ev.dense_backward(dy.cuda(), xd, w.cuda(), name, None if name == "none" else z.cuda())
    for g, (want, tol), what in zip(got, ref, ("dx", "dw", "db")):
        close(g, want, tol, what)
    # each alone gives the same bits
    for i, what in enumerate("xwb"):
        alone = ev.dense_backward(dy.cuda(), xd, w.cuda(), name, None if name == "none" else z.cuda(), want=(what,))
        assert [a is not None for a in alone] == [k == i for k in range(3)] and torch.equal(alone[i], got[i])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 65536, 40), (5, 24, 65536), (600, 20001, 9), (300, 9, 20001)])
@pytest.mark.parametrize("name,kept", [("relu", True), ("gelu", False)])
def test_dense_of_the_widest_layers(B, ev, dtype, shape, name, kept):
    test_dense(ev, dtype, shape, name)
    test_dense_backward(B, ev, dtype, shape, name, kept)


@pytest.mark.parametrize("shape", [(1, 256, 256), (3, 5, 7), (17, 384, 128), (127, 129, 131), (515, 40, 24), (64, 1031, 8), (9001, 201, 139), (2203, 513, 8),
                                   (40001, 4, 8), (17003, 65, 40), (8200, 256, 256), (33001, 24, 32), (12000, 300, 520)])
@pytest.mark.parametrize("name,kept", [("gelu", False), ("silu", True)])
def test_dense_backward_holds_dz_in_16_bits(B, ev, shape, name, kept):
    """bf16 and a smooth activation: dx and dw are off by their own rounding and what fp32 would be off by, unless the caller
    has dz rounded."""
    t, (rows, K, N) = torch.bfloat16, shape
    x, w, dy, z = rand(1, rows, K).to(t), (rand(2, K, N) / math.sqrt(K)).to(t), rand(3, rows, N).to(t), rand(4, rows, N).to(t)
    xd = x.cuda()
    if kept:
        xd = ev.keep_rows(xd)
        x = ev.restore_rows(xd, torch.float32).cpu()
    d = dy.double()
    dz = d * slope(z.double(), name)
    # evaluating the slope as in fp32; the second number's own rounding, 2^-8 of 2^-8
    edz = d.abs() * 16 * U * (1 + z.double().abs()) + 2.0 ** -16 * dz.abs()
    aw, ax = w.double().abs(), x.double().abs()
    dx, dw = dz @ w.double().t(), x.double().t() @ dz
    # two instructions per 16 indices
    tx = edz @ aw.t() + (3 * 2 * (N // 16 + 1) + 2) * U * (dz.abs() @ aw.t()) + (R(t) + U) * dx.abs()
    sections = 2 * 3 * (rows // 128 + 96) + 4              # a slab's instructions (of eight slabs at least), then the slabs
    tw = ax.t() @ edz + sections * U * (ax.t() @ dz.abs()) + (R(t) + U) * dw.abs()
    got = ev.dense_backward(dy.cuda(), xd, w.cuda(), name, z.cuda())
    close(got[0], dx, tx, "dx")
    close(got[1], dw, tw, "dw")
    less = ev.dense_backward(dy.cuda(), xd, w.cuda(), name, z.cuda(), round_dz=True)
    for a, (want, tol), what in zip(less, backward_reference(dy, x, w, z, name, t), ("dx", "dw", "db")):
        close(a, want, tol, what)
    assert torch.equal(less[2], got[2])
    # the other calls do not go by it
    for other, u in ((name, torch.float32), ("relu", t), ("none", t)):
        args = [dy.to(u).cuda(), xd if kept else xd.to(u), w.to(u).cuda(), other, None if other == "none" else z.to(u).cuda()]
        assert all(torch.equal(a, b) for a, b in zip(ev.dense_backward(*args), ev.dense_backward(*args, round_dz=True)))


@pytest.mark.parametrize("rows", [40, 9000])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan, "largest"])
def test_dense_backward_of_what_is_not_finite_in_two_numbers(ev, rows, bad):
    """A gradient that is not finite, or rounds to what is not, reaches its row of dx and its column of dw as with one number."""
    t, K, N = torch.bfloat16, 64, 32
    x, w, dy = rand(1, rows, K).to(t).cuda(), (1 + rand(2, K, N).abs()).to(t).cuda(), rand(3, rows, N).to(t).cuda()
    z = torch.full((rows, N), 30.0, dtype=t, device="cuda")             # a slope of one
    dy[7, 5] = torch.finfo(t).max if bad == "largest" else bad
    if bad == "largest":
        z[7, 5] = 1.2890625                                              # a slope of 1.0023: 3.397e38, which bf16 does not have
    whole, rounded = (ev.dense_backward(dy, x, w, "silu", z, round_dz=r) for r in (False, True))
    for a, b in zip(whole, rounded):
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.isinf(a), torch.isinf(b))
        assert torch.equal(a[torch.isinf(a)], b[torch.isinf(b)])
    fine = torch.ones(rows, dtype=torch.bool)
    fine[7] = False
    assert torch.isfinite(whole[0][fine]).all() and not torch.isfinite(whole[0][7]).any()


def test_dense_backward_refuses_an_unknown_dz(B, ev):
    x = torch.zeros(4, 8, device="cuda")
    w, dw, ws = torch.zeros(8, 8, device="cuda"), torch.zeros(8, 8, device="cuda"), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    args = dict(dtype=B.DC_BF16, act=3, rows=4, n_in=8, n_out=8, dY=x.data_ptr(), lddy=8, Z=x.data_ptr(), ldz=8, X=x.data_ptr(), ldx=8,
                W=w.data_ptr(), ldw=8, dW=dw.data_ptr(), lddw=8, workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    for dz in (-1, 2):
        assert B.dc_dense_backward(ev.ctx, B.DcDenseBackwardArgs(**args, dz=dz)) == B.DC_ERR_INVALID_ARG
        assert "DC_DZ" in B.dc_last_error(ev.ctx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(33001, 24, 32), (9001, 201, 139), (4501, 255, 70), (7003, 131, 129), (3001, 390, 1031), (2203, 513, 8),
                                   (40001, 4, 8), (17003, 65, 40), (9007, 129, 33), (8200, 256, 256), (4100, 260, 9)])
@pytest.mark.parametrize("name,kept", [("relu", False), ("relu", True), ("gelu", True)])
def test_dense_backward_of_many_rows(B, ev, dtype, shape, name, kept):
    test_dense_backward(B, ev, dtype, shape, name, kept)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,first", [(0, 1), (3, 0), (8, 8)])
def test_dense_backward_rows_anywhere(ev, dtype, ld, first):
    t, rows, K, N = TYPES[dtype], 170, 72, 40
    x, w, dy, z = rand(1, rows, K).to(t), (rand(2, K, N) / math.sqrt(K)).to(t), rand(3, rows, N).to(t), rand(4, rows, N).to(t)
    ref = backward_reference(dy, x, w, z, "silu", t)
    got = ev.dense_backward(off_grid(dy, N + ld, first), off_grid(x, K + ld, first), off_grid(w, N + ld, first), "silu",
                            off_grid(z, N + ld, first))
    for g, (want, tol), what in zip(got, ref, ("dx", "dw", "db")):
        close(g, want, tol, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense_backward_keeps_sums_apart(ev, dtype):
    """An infinite gradient reaches its own row of dx, its own columns of dw and db, and nothing else."""
    t, rows, K, N = TYPES[dtype], 600, 64, 48
    x, w, dy = rand(1, rows, K).abs().to(t) + 0.1, (rand(2, K, N).abs() + 0.1).to(t), rand(3, rows, N).to(t)
    clean = ev.dense_backward(dy.cuda(), x.cuda(), w.cuda())
    dy[11, 3] = math.inf
    dx, dw, db = ev.dense_backward(dy.cuda(), x.cuda(), w.cuda())
    assert torch.isinf(dx[11]).all() and torch.isinf(dw[:, 3]).all() and torch.isinf(db[3])
    row, col = torch.arange(rows, device="cuda") != 11, torch.arange(N, device="cuda") != 3
    assert torch.equal(dx[row], clean[0][row]) and torch.equal(dw[:, col], clean[1][:, col]) and torch.equal(db[col], clean[2][col])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense_backward_of_many_rows_keeps_sums_apart(ev, dtype):
    t, rows, K, N = TYPES[dtype], 20001, 70, 48
    x, w, dy = rand(1, rows, K).abs().to(t) + 0.1, (rand(2, K, N).abs() + 0.1).to(t), rand(3, rows, N).to(t)
    z = torch.ones(rows, N, dtype=t)
    clean = ev.dense_backward(dy.cuda(), x.cuda(), w.cuda(), "relu", z.cuda())
    dy[11111, 3] = math.inf
    dx, dw, db = ev.dense_backward(dy.cuda(), x.cuda(), w.cuda(), "relu", z.cuda())
    assert torch.isinf(dx[11111]).all() and torch.isinf(dw[:, 3]).all() and torch.isinf(db[3])
    row, col = torch.arange(rows, device="cuda") != 11111, torch.arange(N, device="cuda") != 3
    assert torch.equal(dx[row], clean[0][row]) and torch.equal(dw[:, col], clean[1][:, col]) and torch.equal(db[col], clean[2][col])


# ---------------------------------------------------------------------------
# kept rows
# ---------------------------------------------------------------------------
def keep_reference(x):
    """Codes and exponent codes by integer search: the smallest exponent whose 127 steps reach the block's largest."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    code, exponent = np.zeros((rows, 32 * nb), np.int8), np.zeros((rows, nb), np.uint8)
    for r, b in itertools.product(range(rows), range(nb)):
        v = x[r, 32 * b:32 * b + 32].astype(np.float64)
        if not np.isfinite(v).all():
            exponent[r, b] = 255
            continue
        m = np.abs(v).max()
        e = -126
        while e < 121 and m > 127 * 2.0 ** e:
            e += 1
        q = np.clip(np.rint(v / 2.0 ** e), -127, 127)
        q[(q == 0) & (v != 0)] = np.sign(v[(q == 0) & (v != 0)])
        code[r, 32 * b:32 * b + 32][:len(v)] = q
        exponent[r, b] = e + 127
    return code, exponent


def kept_values(code, exponent, cols):
    e = np.repeat(exponent.astype(np.float64), 32, 1)
    v = code * np.exp2(e - 127)
    v[e == 255] = np.nan
    return v[:, :cols]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (65, 64), (7, 139), (130, 256), (2, 31)])
@pytest.mark.parametrize("values", ["normal", "wide", "edges", "bad"])
def test_keep_and_restore(ev, dtype, rows, cols, values):
    t = TYPES[dtype]
    x = rand(rows * cols, rows, cols)
    if values == "wide":
        x = x * torch.exp2(torch.from_numpy(np.random.default_rng(3).integers(-160, 120, (rows, cols)).astype(np.float64)))
    x = x.float()
    if values == "edges":
        special = torch.tensor([0.0, -0.0, 1e-45, -1e-45, 1.1754944e-38, 127.0, 127.5, 126.99999, 63.5, 1.984375, 1.9843751, 3.4028235e38,
                                -3.4028235e38, 0.5, -0.5, 0.25])
        x = special[torch.from_numpy(np.random.default_rng(5).integers(0, len(special), (rows, cols)))]
        if rows > 2:
            x[1] = 0.0
            x[2] = torch.where(x[2].abs() > 1e38, torch.ones(()), x[2])
    if values == "bad":
        x[0, 0] = math.inf
        x[rows - 1, cols - 1] = math.nan
    x = x.to(t)
    code, exponent = keep_reference(x.float().numpy())
    k = ev.keep_rows(x.cuda())
    assert np.array_equal(k.code.cpu().numpy(), code) and np.array_equal(k.exponent.cpu().numpy(), exponent)
    want = kept_values(code, exponent, cols)
    for out in (torch.float32, torch.bfloat16):           # a kept value is a bf16 number
        got = ev.restore_rows(k, out).double().cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True)
    xs = x.double().numpy()
    ok = np.isfinite(want)
    assert np.array_equal(np.sign(want[ok]), np.sign(xs[ok]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld,first", [(1, 0), (0, 3), (16, 16)])
def test_keep_rows_anywhere(B, ev, dtype, ld, first):
    t, rows, cols = TYPES[dtype], 37, 96
    x = rand(2, rows, cols).to(t)
    code, exponent = keep_reference(x.float().numpy())
    k = ev.keep_rows(off_grid(x, cols + ld, first))
    assert np.array_equal(k.code.cpu().numpy(), code) and np.array_equal(k.exponent.cpu().numpy(), exponent)
    wide = torch.zeros(rows, cols + 7, dtype=torch.int8, device="cuda")
    wide[:, :cols] = k.code
    k2 = B.KeptRows(wide[:, :cols], k.exponent, cols)
    out = off_grid(torch.zeros(rows, cols, dtype=t), cols + ld, first)
    assert np.array_equal(ev.restore_rows(k2, t, out=out).double().cpu().numpy(), kept_values(code, exponent, cols))


@pytest.mark.parametrize("rows", [1, 37])
def test_kept_rows_in_c_calls(B, ev, rows):
    """The struct of kept rows, of those that keep_rows made and of those put together from tensors."""
    cols = 72
    x = rand(3, rows, cols).float().cuda()
    k = ev.keep_rows(x)
    wide = torch.zeros(rows, 128, dtype=torch.int8, device="cuda")
    wide[:, :96] = k.code
    want = ev.restore_rows(k)
    for kept in (k, B.KeptRows(k.code, k.exponent, cols), B.KeptRows(wide[:, :96], k.exponent, cols)):
        out = torch.empty_like(x)
        assert B.dc_restore_rows(ev.ctx, B.DC_F32, rows, cols, kept.c, out.data_ptr(), cols, torch.cuda.current_stream().cuda_stream) == B.DC_OK
        assert torch.equal(out, want)


# ---------------------------------------------------------------------------
# graph norm
# ---------------------------------------------------------------------------
EPS = 1e-5
# rows per graph: none, one, many short, one that the workgroup does not hold, long ones that are split, next to short ones
RAGGED = {"one": [1], "short": [0, 1, 2, 0, 9, 30, 3, 1, 0], "module": [729], "many": [5, 11, 0, 7] * 300, "middle": [300, 40, 650, 0, 1],
          "long": [5000, 3, 0, 2600, 1, 9000, 17], "empty": [0, 0, 0]}
GROUPS = [(128, 4), (256, 8), (32, 32), (24, 1), (36, 9), (35, 5), (6, 2), (512, 1)]


def norm_statistics(x, sizes, G):
    """mean and variance [graphs, G] in 64 bits."""
    C = x.shape[1]
    mean, var = torch.zeros(len(sizes), G, dtype=torch.float64), torch.zeros(len(sizes), G, dtype=torch.float64)
    lo = 0
    for i, n in enumerate(sizes):
        if n:
            v = x[lo:lo + n].double().view(n, G, C // G)
            mean[i] = v.mean((0, 2))
            var[i] = ((v - mean[i][None, :, None]) ** 2).mean((0, 2))
        lo += n
    return mean, var


def per_row(v, sizes, C):
    """[graphs, G] -> [rows, C]"""
    return torch.repeat_interleave(v, torch.tensor(sizes), 0).repeat_interleave(C // v.shape[1], 1)


def offsets(sizes, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(sizes)]), dtype=torch.int32, device="cuda")


def norm_inputs(sizes, C, dtype, seed=1):
    x = rand(seed, sum(sizes), C) * (0.5 + rand(seed + 1, C).abs()) + 2 * rand(seed + 2, C)
    return x.to(TYPES[dtype]), (1 + 0.2 * rand(seed + 3, C)).float(), (0.2 * rand(seed + 4, C)).float()


def check_norm(ev, x, sizes, G, gamma, beta, name, dtype, got):
    t, C = TYPES[dtype], x.shape[1]
    y, mean, rstd = got
    mu, var = norm_statistics(x, sizes, G)
    rs = 1 / torch.sqrt(var + EPS)
    # sums in 64 bits, each statistic rounded once; the variance as a difference of 64-bit numbers
    close(mean, mu, 2 * U * mu.abs() + 1e-12, "mean")
    close(rstd, rs, 4 * U * rs + rs * 1e-13 * (mu * mu + var) / (var + EPS), "rstd")
    m, r = per_row(mu, sizes, C), per_row(rs, sizes, C)
    d = x.double() - m
    z = gamma.double() * d * r + beta.double()
    ez = gamma.double().abs() * r * (2 * U * m.abs() + 8 * U * d.abs()) + 2 * U * (z.abs() + beta.double().abs())
    want = act(z, name)
    close(y, want, 1.13 * ez + 8 * U * z.abs() + (R(t) + U) * want.abs(), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", list(RAGGED))
@pytest.mark.parametrize("C,G", GROUPS)
def test_graph_norm(ev, dtype, sizes, C, G):
    s = RAGGED[sizes]
    print(dtype, sizes, C, G, flush=True)
    x, gamma, beta = norm_inputs(s, C, dtype)
    name = ["none", "relu", "silu", "gelu"][(C + len(s)) % 4]
    got = ev.graph_norm(x.cuda(), offsets(s), G, gamma.cuda(), beta.cuda(), EPS, name)
    check_norm(ev, x, s, G, gamma, beta, name, dtype, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", ["short", "middle", "long"])
def test_graph_norm_rows_anywhere(ev, dtype, sizes):
    """Rows apart, in place, and rows of no graph in front and behind that stay as they are; no gamma and beta."""
    s, C, G, t = RAGGED[sizes], 48, 6, TYPES[dtype]
    x, _, _ = norm_inputs(s, C, dtype)
    n = x.shape[0]
    padded = torch.full((n + 8, C), 7.0, dtype=t)
    padded[3:3 + n] = x
    v = off_grid(padded, C + 5, 1)
    got, mean, rstd = ev.graph_norm(v, offsets(s, 3), G, act="silu", eps=EPS, out=v)
    check_norm(ev, x, s, G, torch.ones(C), torch.zeros(C), "silu", dtype, (got[3:3 + n], mean, rstd))
    assert (got[:3] == 7).all() and (got[3 + n:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph_norm_large_offset(ev, dtype):
    """Values far from zero next to their spread, and a group that is constant."""
    s, C, G = [700, 3, 4000], 32, 4
    x = (1000 + rand(1, sum(s), C)).to(TYPES[dtype])
    x[700:703, :8] = 5.0
    got = ev.graph_norm(x.cuda(), offsets(s), G, None, None, EPS)
    check_norm(ev, x, s, G, torch.ones(C), torch.zeros(C), "none", dtype, got)
    assert not got[0][700:703, :8].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,spread", [(1e5, 1.0), (1e6, 0.1), (1e7, 1.0), (-1e8, 8.0)])
@pytest.mark.parametrize("sizes", [[9] * 300 + [0, 1, 40], [300, 700, 2, 1000], [5000, 3, 9000]], ids=["waves", "held", "chunks"])
def test_graph_norm_far_from_zero(ev, dtype, offset, spread, sizes):
    """Values that lie up to 2^23 times their spread from zero, and a group that is constant: the statistics and the result
    are off by roundings of their own size, whatever the offset."""
    C, G, t = 32, 4, TYPES[dtype]
    x = (offset * (1 + 1e-8 * rand(6, C)) + spread * rand(5, sum(sizes), C)).to(t)
    x[:, 8:16] = 123456.7
    gamma, beta = (1 + 0.2 * rand(7, C)).float(), (0.2 * rand(8, C)).float()
    xd, off = x.cuda(), offsets(sizes)
    y, mean, rstd = ev.graph_norm(xd, off, G, gamma.cuda(), beta.cuda(), EPS, "silu")
    mu, var = norm_statistics(x, sizes, G)
    rs = 1 / torch.sqrt(var + EPS)
    # 64-bit sums over m values, counted from the first one, x0: m roundings of 2^-53 of their size at most
    first = torch.tensor(np.minimum(np.concatenate([[0], np.cumsum(sizes)])[:-1], sum(sizes) - 1))
    far = var + (x[first][:, ::C // G].double() - mu) ** 2
    sums = 4 * max(sizes) * (C // G) * 2.0 ** -53 * far
    filled = torch.tensor([n > 0 for n in sizes])[:, None]
    mu, far, sums = (torch.where(filled, v, torch.zeros_like(v)) for v in (mu, far, sums))
    close(mean, mu, 1.01 * U * mu.abs() + torch.sqrt(sums * 2.0 ** -53), "mean")
    close(rstd, rs, 2 * U * rs + rs * sums / (var + EPS), "rstd")
    m, r = per_row(mu, sizes, C), per_row(rs, sizes, C)
    d = x.double() - m
    z = gamma.double() * d * r + beta.double()
    # x - mu: two roundings of its size, and mu's second part, rounded once
    ez = gamma.double().abs() * r * (8 * U * d.abs() + 4 * U * U * m.abs()) + 2 * U * (z.abs() + beta.double().abs())
    ez = ez + (gamma.double() * d * r).abs() * per_row(sums / (var + EPS), sizes, C)
    want = act(z, "silu")
    close(y, want, 1.13 * ez + 8 * U * z.abs() + (R(t) + U) * want.abs(), "y")
    assert (rstd[:, 1] == rstd[0, 1]).all() and (mean[filled[:, 0].cuda(), 1] == x[0, 8].float().item()).all()
    again = ev.graph_norm(xd, off, G, gamma.cuda(), beta.cuda(), EPS, "silu", out=xd)
    assert all(torch.equal(a, b) for a, b in zip(again, (y, mean, rstd)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_graph_norm_of_what_is_not_finite(ev, dtype, bad):
    """A value that is not finite, a graph's first one among them, reaches its graph and group and nothing else."""
    s, C, G = [9, 40, 5000, 7], 32, 4
    x = rand(3, sum(s), C).to(TYPES[dtype])
    hit = [(0, 0, 0), (9, 1, 8), (30, 1, 16), (49, 2, 0), (4000, 2, 24)]           # row, graph, column
    for row, _, col in hit:
        x[row, col] = bad
    y, mean, rstd = ev.graph_norm(x.cuda(), offsets(s), G, None, None, EPS)
    lost = torch.zeros(len(s), G, dtype=torch.bool)
    for _, g, col in hit:
        lost[g, col // (C // G)] = True
    want = torch.tensor(bad).expand(int(lost.sum()))
    assert torch.equal(mean.cpu()[lost].nan_to_num(nan=7.0), want.nan_to_num(nan=7.0)) and torch.isnan(rstd.cpu()[lost]).all()
    assert torch.isfinite(mean.cpu()[~lost]).all() and torch.isfinite(rstd.cpu()[~lost]).all()
    assert torch.equal(torch.isnan(y).cpu(), per_row(lost, s, C))


def norm_back_reference(x, dy, dres, sizes, G, gamma, beta, mean, rstd, name, t):
    C = x.shape[1]
    g, b = gamma.double(), beta.double()
    m, r = per_row(mean.double(), sizes, C), per_row(rstd.double(), sizes, C)
    d = x.double() - m
    xh = d * r
    e_xh = 3 * U * xh.abs()                               # the statistics are given: subtraction and product
    z = g * xh + b
    k = slope(z, name)
    dz = dy.double() * k
    # the slopes' own slopes are below 1; evaluating one: sixteen roundings of size 1 + |z|
    e_dz = torch.zeros_like(dz) if name in ("none", "relu") else dy.double().abs() * (g.abs() * e_xh + 2 * U * (z.abs() + b.abs()) + 16 * U * (1 + z.abs()))
    e_dz = e_dz + U * dz.abs()
    u, e_u = g * dz, g.abs() * e_dz + U * (g * dz).abs()

    def mean_of(v):
        out = torch.zeros(len(sizes), G, dtype=torch.float64)
        lo = 0
        for i, n in enumerate(sizes):
            if n:
                out[i] = v[lo:lo + n].reshape(n, G, C // G).mean((0, 2))
            lo += n
        return per_row(out, sizes, C)
    s1, s2 = mean_of(u), mean_of(u * xh)
    e1, e2 = mean_of(e_u) + 2 * U * s1.abs(), mean_of(e_u * xh.abs() + u.abs() * e_xh) + 2 * U * s2.abs()
    dx = r * (u - s1 - xh * s2)
    e = r * (e_u + e1 + xh.abs() * e2 + e_xh * s2.abs() + 4 * U * (u.abs() + s1.abs() + (xh * s2).abs()))
    if dres is not None:
        dx = dx + dres.double()
        e = e + U * dx.abs()
    # column sums: a thread's rows of a graph in fp32 (at most 64 here), then 64 bits
    dgamma, dbeta = (dz * xh).sum(0), dz.sum(0)
    eg = (e_dz * xh.abs() + dz.abs() * e_xh).sum(0) + 70 * U * (dz * xh).abs().sum(0)
    eb = e_dz.sum(0) + 70 * U * dz.abs().sum(0)
    return (dx, e + (R(t) + U) * dx.abs()), (dgamma, eg), (dbeta, eb), z


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", list(RAGGED))
@pytest.mark.parametrize("C,G", GROUPS)
def test_graph_norm_backward(ev, dtype, sizes, C, G):
    s, t = RAGGED[sizes], TYPES[dtype]
    x, gamma, beta = norm_inputs(s, C, dtype)
    dy, dres = rand(11, sum(s), C).to(t), rand(12, sum(s), C).to(t)
    i = C + len(s)
    name, kept, res = ["none", "silu", "gelu"][i % 3], i % 2 == 0, dres if i % 4 < 2 else None
    print(dtype, sizes, C, G, name, kept, flush=True)
    off = offsets(s)
    xd = x.cuda()
    _, mean, rstd = ev.graph_norm(xd, off, G, gamma.cuda(), beta.cuda(), EPS, name)
    if kept:
        xd = ev.keep_rows(xd)
        x = ev.restore_rows(xd, torch.float32).cpu()
    ref = norm_back_reference(x, dy, res, s, G, gamma, beta, mean.cpu(), rstd.cpu(), name, t)
    got = ev.graph_norm_backward(dy.cuda(), xd, off, G, gamma.cuda(), beta.cuda(), mean, rstd, name,
                                 None if res is None else res.cuda())
    for g, (want, tol), what in zip(got, ref, ("dx", "dgamma", "dbeta")):
        close(g, want, tol, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,G", [(256, 8), (128, 4)])
def test_graph_norm_vector_gradients_of_a_long_graph_among_short_ones(ev, dtype, C, G):
    """A thousand rows that one wave takes beside thousands of graphs of nine: terms of one sign that a running sum in fp32 rounds
    to the same side each time; dgamma and dbeta are off by at most the 70 roundings of runs of 64 rows."""
    sizes, t = [9] * 1500 + [1000] + [9] * 1500, TYPES[dtype]
    first = 9 * 1500
    x = torch.zeros(sum(sizes), C)
    x[first:first + 1000] = 1 + 2.0 ** -15 - 2.0 ** -22          # a constant xh, below
    dy = torch.zeros(sum(sizes), C)
    dy[first:first + 1000] = 1 + 2.0 ** -15 - 2.0 ** -22
    x, dy = x.to(t), dy.to(t)
    mean, rstd = torch.zeros(len(sizes), G, device="cuda"), torch.ones(len(sizes), G, device="cuda")
    ref = norm_back_reference(x, dy, None, sizes, G, torch.ones(C), torch.zeros(C), mean.cpu(), rstd.cpu(), "none", t)
    got = ev.graph_norm_backward(dy.cuda(), x.cuda(), offsets(sizes), G, None, None, mean, rstd)
    for g, (want, tol), what in zip(got, ref, ("dx", "dgamma", "dbeta")):
        close(g, want, tol, what)


@pytest.mark.parametrize("sizes", ["short", "middle", "long"])
def test_graph_norm_backward_relu_in_place(ev, sizes):
    """ReLU, on inputs whose normalised values are not next to its corner; dx in place of dy, rows of no graph as they were."""
    s, C, G = RAGGED[sizes], 32, 4
    x, gamma, beta = norm_inputs(s, C, "f32", seed=21)
    n, dy = x.shape[0], rand(31, sum(s), C).float()
    pad = lambda v: torch.cat([torch.full((2, C), 7.0), v, torch.full((5, C), 7.0)]).cuda()
    off = offsets(s, 2)
    _, mean, rstd = ev.graph_norm(pad(x), off, G, gamma.cuda(), beta.cuda(), EPS, "relu")
    # a value next to the corner moves away from it
    for _ in range(3):
        z = norm_back_reference(x, dy, None, s, G, gamma, beta, mean.cpu(), rstd.cpu(), "relu", torch.float32)[3]
        x = torch.where(z.abs() < 1e-4, x + 0.01, x)
    ref = norm_back_reference(x, dy, None, s, G, gamma, beta, mean.cpu(), rstd.cpu(), "relu", torch.float32)
    assert ref[3].abs().min() > 1e-5
    buf = pad(dy)
    dx, dgamma, dbeta = ev.graph_norm_backward(buf, pad(x), off, G, gamma.cuda(), beta.cuda(), mean, rstd, "relu", out=buf)
    assert (dx[:2] == 7).all() and (dx[2 + n:] == 7).all()
    for g, (want, tol), what in zip((dx[2:2 + n], dgamma, dbeta), ref, ("dx", "dgamma", "dbeta")):
        close(g, want, tol, what)


def test_graph_norm_reports_bad_offsets(B, ev):
    """Offsets that do not ascend within the rows: those graphs are left alone, the others are done, dc_check tells."""
    C, G = 16, 2
    x = rand(1, 40, C).float().cuda()
    for off in ([0, 10, 5, 40], [0, 10, 41], [-1, 10, 40]):
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        out = torch.full_like(x, 7.0)
        ev.graph_norm(x, o, G, out=out)
        assert ev.check() == B.DC_ERR_BAD_GRAPH
        assert ev.check() == B.DC_OK
        good = [(a, b) for a, b in zip(off, off[1:]) if 0 <= a <= b <= 40]
        touched = torch.zeros(40, dtype=torch.bool)
        for a, b in good:
            touched[a:b] = True
        assert torch.equal((out != 7).any(1).cpu(), touched)


def test_graph_norm_overlapping_long_graphs(B, ev):
    """Offsets that jump back and forth name more long graphs than the rows can hold: reported, nothing outside is touched."""
    C, G, rows = 16, 2, 5000
    x = torch.full((rows + 64, C), 3.0, device="cuda")
    off = torch.tensor([0, rows] * 40, dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    ev.graph_norm(x[:rows], off, G, out=out[:rows])
    ev.graph_norm_backward(x[:rows], x[:rows], off, G, None, None, torch.zeros(79, G, device="cuda"), torch.ones(79, G, device="cuda"))
    assert ev.check() == B.DC_ERR_BAD_GRAPH
    assert (out[rows:] == 7).all()


# ---------------------------------------------------------------------------
# differences, streams, graphs, chains
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("name", ["none", "gelu", "silu"])
def test_gradients_against_differences(ev, name):
    """The gradient along a direction is the difference quotient of the forward pass along it: off by h^2 / 6 of the third
    derivative, and by the forward's rounding over h."""
    s, C, G, N, h = [30, 1, 9, 200], 32, 4, 24, 2.0 ** -7
    x, gamma, beta = norm_inputs(s, C, "f32")
    x = x / 2
    off, w, b = offsets(s), (rand(7, C, N) / math.sqrt(C)).float().cuda(), rand(8, N).float().cuda()
    gy = rand(9, sum(s), N).float().cuda()

    def value(xx, gg, ww):
        u, mean, rstd = ev.graph_norm(xx, off, G, gg, beta.cuda(), 0.1, name)
        y, pre = ev.dense(u, ww, b, name, want_pre=True)
        return float((y.double() * gy.double()).sum()), (u, mean, rstd, pre)
    xd, gd = x.cuda(), gamma.cuda()
    _, (u, mean, rstd, pre) = value(xd, gd, w)
    du, dw, db = ev.dense_backward(gy, u, w, name, pre)
    dx, dgamma, dbeta = ev.graph_norm_backward(du, xd, off, G, gd, beta.cuda(), mean, rstd, name)
    for v, grad, which in ((xd, dx, 0), (gd, dgamma, 1), (w, dw, 2)):
        d = rand(40 + which, *v.shape).float().cuda()
        d = d / d.norm()
        args = [xd, gd, w]
        args[which] = v + h * d
        up = value(*args)[0]
        args[which] = v - h * d
        down = value(*args)[0]
        want = float((grad.double() * d.double()).sum())
        # the direction has length 1: third derivatives of the sum stay below its gradient's size times 16; the forward's
        # 5760 outputs of size about 1 are off by some 100 U each, at random
        tol = 16 * h * h / 6 * float(grad.norm()) + 100 * U * math.sqrt(sum(s) * N) * 4 / h
        assert abs((up - down) / (2 * h) - want) <= tol, (which, (up - down) / (2 * h), want, tol)


def test_operators_on_another_stream_and_in_a_graph(ev):
    """A training pass of two operators on a stream of its own, captured and replayed with eager work in between."""
    s, C, G, N = [900, 2, 0, 1700, 40] * 3, 64, 4, 96
    x, gamma, beta = norm_inputs(s, C, "f32")
    off, w, b = offsets(s), (rand(7, C, N) / 8).float().cuda(), rand(8, N).float().cuda()
    xs, gd, bd, gy = x.cuda(), gamma.cuda(), beta.cuda(), rand(9, sum(s), N).float().cuda()

    def step():
        u, mean, rstd = ev.graph_norm(xs, off, G, gd, bd, EPS, "silu")
        k = ev.keep_rows(xs)
        y, pre = ev.dense(u, w, b, "gelu", want_pre=True)
        du, dw, db = ev.dense_backward(gy, u, w, "gelu", pre)
        return (y, dw, db) + ev.graph_norm_backward(du, k, off, G, gd, bd, mean, rstd, "silu", residual=du)
    first = [v.clone() for v in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graphs = []
    for _ in range(2):                                    # two graphs, each with workspaces of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for k in range(4):
        xs.copy_(x.cuda() * (1 + k))
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = step()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), k


def test_bf16_gradients_in_a_graph(ev):
    """dz in two numbers and in one, and a norm far from zero, captured together and replayed with eager work in between."""
    s, C, G, N, t = [900, 2, 0, 1700, 40] * 2, 64, 4, 96, torch.bfloat16
    x, gamma, beta = norm_inputs(s, C, "bf16")
    off, w, gy = offsets(s), (rand(7, C, N) / 8).to(t).cuda(), rand(9, sum(s), N).to(t).cuda()
    xs, gd, bd = x.cuda(), gamma.cuda(), beta.cuda()

    def step():
        u, mean, rstd = ev.graph_norm(xs, off, G, gd, bd, EPS, "silu")
        _, pre = ev.dense(u, w, None, "gelu", want_pre=True)
        out = (mean, rstd)
        for rounded in (False, True):
            du, dw, db = ev.dense_backward(gy, u, w, "gelu", pre, round_dz=rounded)
            out += (dw, db) + ev.graph_norm_backward(du, xs, off, G, gd, bd, mean, rstd, "silu")
        return out
    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for k in range(4):
        xs.copy_(x.cuda() * (1 + k) + 50 * k)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), k
        torch.cuda.synchronize()


def test_results_do_not_depend_on_what_else_is_there(ev):
    """The same call twice, and the rows of a graph next to other graphs: the same bits."""
    s, C, G = [40, 700, 3, 5000], 64, 8
    x, gamma, beta = norm_inputs(s, C, "bf16")
    dy = rand(9, sum(s), C).bfloat16().cuda()
    off = offsets(s)
    a = ev.graph_norm(x.cuda(), off, G, gamma.cuda(), beta.cuda(), EPS, "gelu")
    b = ev.graph_norm(x.cuda(), off, G, gamma.cuda(), beta.cuda(), EPS, "gelu")
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    p = ev.graph_norm_backward(dy, x.cuda(), off, G, gamma.cuda(), beta.cuda(), a[1], a[2], "gelu")
    q = ev.graph_norm_backward(dy, x.cuda(), off, G, gamma.cuda(), beta.cuda(), a[1], a[2], "gelu")
    assert all(torch.equal(u, v) for u, v in zip(p, q))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,G", [(208, 16), (36, 9), (24, 1), (512, 8)])
def test_graph_norm_of_many_long_graphs(ev, dtype, C, G):
    """More long graphs than the last wave of a row of channels has channels."""
    s = [4100 + 61 * i for i in range(70)] if C < 40 else [4200 + 353 * i for i in range(22)]
    x, gamma, beta = norm_inputs(s, C, dtype)
    off = offsets(s)
    got = ev.graph_norm(x.cuda(), off, G, gamma.cuda(), beta.cuda(), EPS, "silu")
    check_norm(ev, x, s, G, gamma, beta, "silu", dtype, got)
    dy = rand(9, sum(s), C).to(TYPES[dtype])
    ref = norm_back_reference(x, dy, None, s, G, gamma, beta, got[1].cpu(), got[2].cpu(), "silu", TYPES[dtype])
    back = ev.graph_norm_backward(dy.cuda(), x.cuda(), off, G, gamma.cuda(), beta.cuda(), got[1], got[2], "silu")
    for g, (want, tol), what in zip(back, ref, ("dx", "dgamma", "dbeta")):
        close(g, want, tol, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,C,G", [([30, 31, 0, 40] * 25, 512, 8), ([30, 31, 0, 40] * 25, 468, 52), ([110, 131, 1] * 700, 75, 5), ([100] * 1030, 104, 8)])
def test_graph_norm_in_slabs_of_waves(ev, dtype, sizes, C, G):
    """Rows wider than a wave's vectors, and graphs of more rows than a wave holds of them."""
    x, gamma, beta = norm_inputs(sizes, C, dtype)
    off = offsets(sizes)
    got = ev.graph_norm(x.cuda(), off, G, gamma.cuda(), beta.cuda(), EPS, "gelu")
    check_norm(ev, x, sizes, G, gamma, beta, "gelu", dtype, got)
    dy, dres = rand(9, sum(sizes), C).to(TYPES[dtype]), rand(10, sum(sizes), C).to(TYPES[dtype])
    ref = norm_back_reference(x, dy, dres, sizes, G, gamma, beta, got[1].cpu(), got[2].cpu(), "gelu", TYPES[dtype])
    back = ev.graph_norm_backward(dy.cuda(), x.cuda(), off, G, gamma.cuda(), beta.cuda(), got[1], got[2], "gelu", dres.cuda())
    for g, (want, tol), what in zip(back, ref, ("dx", "dgamma", "dbeta")):
        close(g, want, tol, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("C,G", [(8192, 16), (8184, 24), (1023, 3), (2048, 2048)])
def test_graph_norm_of_wide_rows(ev, dtype, C, G, odd):
    """Channels up to the most there may be, groups of one channel to 512; rows that no vector of channels fits (odd)."""
    sizes, t = [3, 0, 1300, 40], TYPES[dtype]
    x, gamma, beta = norm_inputs(sizes, C, dtype)
    off, ld = offsets(sizes), C + (5 if odd else 0)
    place = lambda v: off_grid(v, ld, 1 if odd else 0)
    got = ev.graph_norm(place(x), off, G, gamma.cuda(), beta.cuda(), EPS, "silu", out=place(x))
    check_norm(ev, x, sizes, G, gamma, beta, "silu", dtype, got)
    dy = rand(9, sum(sizes), C).to(t)
    ref = norm_back_reference(x, dy, None, sizes, G, gamma, beta, got[1].cpu(), got[2].cpu(), "silu", t)
    back = ev.graph_norm_backward(place(dy), place(x), off, G, gamma.cuda(), beta.cuda(), got[1], got[2], "silu", out=place(dy))
    for g, (want, tol), what in zip(back, ref, ("dx", "dgamma", "dbeta")):
        close(g, want, tol, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph_norm_gradients_of_many_long_graphs_repeat(ev, dtype):
    """Graphs that are cut into chunks are found in any order; the sums over them are formed in theirs."""
    s, C, G = [5000 + 137 * i for i in range(40)] + [3, 0, 9000], 32, 4
    x, gamma, beta = norm_inputs(s, C, dtype)
    dy, off = rand(9, sum(s), C).to(TYPES[dtype]).cuda(), offsets(s)
    x, gamma, beta = x.cuda(), gamma.cuda(), beta.cuda()
    _, mean, rstd = ev.graph_norm(x, off, G, gamma, beta, EPS, "silu")
    first = ev.graph_norm_backward(dy, x, off, G, gamma, beta, mean, rstd, "silu")
    for _ in range(20):
        again = ev.graph_norm_backward(dy, x, off, G, gamma, beta, mean, rstd, "silu")
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_offsets_beyond_32_bits(ev):
    """Arrays of more than 4 GiB: the last rows against 64 bits, everything that is summed over all rows too."""
    rows, C, G, per = 8_600_000, 128, 4, 1000
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(rows, C, generator=g, device="cuda")
    w = torch.randn(C, C, generator=g, device="cuda") / math.sqrt(C)
    last = slice(rows - per, rows)
    tail, wc = x[last].cpu(), w.cpu()
    y = ev.dense(x, w, act="silu")
    _, _, want, tol = dense_reference(tail, wc, None, None, "silu", torch.float32)
    close(y[last], want, tol, "dense")
    # gradients: y serves as dy
    dx, dw, db = ev.dense_backward(y, x, w)
    dy = y[last].cpu()
    (rx, tx), _, _ = backward_reference(dy, tail, wc, None, "none", torch.float32)
    close(dx[last], rx, tx, "dx")
    del dx
    rw, aw, rb, ab = (torch.zeros(s, dtype=torch.float64, device="cuda") for s in ((C, C), (C, C), (C,), (C,)))
    for lo in range(0, rows, 1_000_000):
        a, d = x[lo:lo + 1_000_000].double(), y[lo:lo + 1_000_000].double()
        rw += a.t().contiguous() @ d
        aw += a.abs().t().contiguous() @ d.abs()
        rb += d.sum(0)
        ab += d.abs().sum(0)
    sections = 3 * 96 + rows // (64 * 128) + 4              # of a slab, of which there are at least 128 here
    close(dw, rw.cpu(), (sections * U * aw + 2 * U * rw.abs()).cpu(), "dw")
    close(db, rb.cpu(), (4 * U * ab).cpu(), "db")
    # norms of graphs of 1000 rows, then rows in 8 bits
    off = torch.arange(0, rows + 1, per, dtype=torch.int32, device="cuda")
    out, mean, rstd = ev.graph_norm(x, off, G, eps=EPS, act="silu", out=y)
    one = torch.ones(C), torch.zeros(C)
    check_norm(ev, tail, [per], G, *one, "silu", "f32", (out[last], mean[-1:], rstd[-1:]))
    ref = norm_back_reference(tail, tail, None, [per], G, *one, mean[-1:].cpu(), rstd[-1:].cpu(), "silu", torch.float32)
    back = ev.graph_norm_backward(x, x, off, G, None, None, mean, rstd, "silu", out=y)
    close((back[0] if isinstance(back, tuple) else back)[last], *ref[0][:2], "dx of the norm")
    kept = ev.keep_rows(x)
    ev.restore_rows(kept, out=y)
    assert torch.equal(y[last], ev.restore_rows(ev.keep_rows(x[last])))


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("rows,graphs,C,G", [(66559, 1, 32, 4), (66559, 3, 490, 1), (65617, 29, 175, 1), (65638, 388, 366, 1), (300, 7, 64, 8)])
def test_graph_norm_stays_in_its_workspace(B, ev, rows, graphs, C, G):
    """A workspace of just the bytes asked for, between others that stay as they are; rows where a CU's four chunks come
    out a little shorter than a fourth of its share."""
    x, dy = rand(1, rows, C).float().cuda(), rand(2, rows, C).float().cuda()
    out, dx, stats, vectors = torch.empty_like(x), torch.empty_like(x), torch.empty(2, graphs, G, device="cuda"), torch.empty(2, C, device="cuda")
    cut = np.linspace(0, rows, graphs + 1).astype(np.int64)
    off = torch.tensor(cut, dtype=torch.int32, device="cuda")
    args = dict(dtype=B.DC_F32, act=3, rows=rows, n_graphs=graphs, channels=C, groups=G, eps=1e-5, node_off=off.data_ptr(),
                X=x.data_ptr(), ldx=C, mean=stats[0].data_ptr(), rstd=stats[1].data_ptr(), Y=out.data_ptr(), ldy=C, dY=dy.data_ptr(), lddy=C,
                dX=dx.data_ptr(), lddx=C, dgamma=vectors[0].data_ptr(), dbeta=vectors[1].data_ptr())
    for back, call in ((False, B.dc_graph_norm), (True, B.dc_graph_norm_backward)):
        size = B.dc_graph_norm_bytes(ev.ctx, rows, graphs, C, G, back)
        buf = torch.full((size + (4 << 20),), 77, dtype=torch.uint8, device="cuda")
        ws = buf[2 << 20:(2 << 20) + size]
        torch.cuda.synchronize()
        assert call(ev.ctx, B.DcGraphNormArgs(**args, workspace=ws.data_ptr(), workspace_bytes=size)) == B.DC_OK
        torch.cuda.synchronize()
        assert ev.check() == B.DC_OK
        assert (buf[:2 << 20] == 77).all() and (buf[(2 << 20) + size:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (5000, 96, 139), (9001, 257, 256), (257, 700, 33)])
def test_dense_backward_stays_in_its_workspace(B, ev, dtype, act, rows, K, N):
    t, code = TYPES[dtype], B.DC_F32 if dtype == "f32" else B.DC_BF16
    x, w, dy, z = (rand(i, *s).to(t).cuda() for i, s in enumerate([(rows, K), (K, N), (rows, N), (rows, N)], 1))
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device="cuda")
    size = B.dc_dense_backward_bytes(ev.ctx, code, act, rows, K, N)
    buf = torch.full((size + (4 << 20),), 77, dtype=torch.uint8, device="cuda")
    ws = buf[2 << 20:(2 << 20) + size]
    torch.cuda.synchronize()
    assert B.dc_dense_backward(ev.ctx, B.DcDenseBackwardArgs(
        dtype=code, act=act, rows=rows, n_in=K, n_out=N, dY=dy.data_ptr(), lddy=N, Z=z.data_ptr(), ldz=N, X=x.data_ptr(), ldx=K,
        W=w.data_ptr(), ldw=N, dX=dx.data_ptr(), lddx=K, dW=dw.data_ptr(), lddw=N, db=db.data_ptr(), workspace=ws.data_ptr(),
        workspace_bytes=size)) == B.DC_OK
    torch.cuda.synchronize()
    assert (buf[:2 << 20] == 77).all() and (buf[(2 << 20) + size:] == 77).all()


def test_c_calls_refuse_arrays_in_each_others_place_and_rows_too_far_apart(B, ev):
    """Each refused with nothing enqueued: what a kernel would still read, or offsets beyond what it counts in."""
    x, w, y, z = (torch.zeros(8, 8, device="cuda") for _ in range(4))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    ok = dict(dtype=B.DC_F32, act=1, rows=8, n_in=8, n_out=8, X=x.data_ptr(), ldx=8, W=w.data_ptr(), ldw=8, Z=z.data_ptr(), ldz=8,
              Y=y.data_ptr(), ldy=8)
    far = (1 << 22) + 1
    for bad, want in [(dict(Y=x.data_ptr()), B.DC_ERR_INVALID_ARG), (dict(Z=x.data_ptr()), B.DC_ERR_INVALID_ARG),
                      (dict(Z=y.data_ptr()), B.DC_ERR_INVALID_ARG), (dict(residual=z.data_ptr(), ld_residual=8), B.DC_ERR_INVALID_ARG),
                      (dict(ldx=far), B.DC_ERR_UNSUPPORTED), (dict(ldw=far), B.DC_ERR_UNSUPPORTED), (dict(ldy=far), B.DC_ERR_UNSUPPORTED),
                      (dict(ldz=far), B.DC_ERR_UNSUPPORTED)]:
        assert B.dc_dense(ev.ctx, B.DcDenseArgs(**{**ok, **bad})) == want, bad
    back = dict(dtype=B.DC_F32, act=1, rows=8, n_in=8, n_out=8, dY=y.data_ptr(), lddy=8, Z=z.data_ptr(), ldz=8, X=x.data_ptr(), ldx=8,
                W=w.data_ptr(), ldw=8, dX=ws.data_ptr(), lddx=8, dW=ws.data_ptr() + 4096, lddw=8, workspace=ws.data_ptr() + 8192,
                workspace_bytes=ws.numel() - 8192)
    for bad, want in [(dict(dX=y.data_ptr()), B.DC_ERR_INVALID_ARG), (dict(dX=z.data_ptr()), B.DC_ERR_INVALID_ARG),
                      (dict(dX=x.data_ptr()), B.DC_ERR_INVALID_ARG), (dict(lddx=far), B.DC_ERR_UNSUPPORTED)]:
        assert B.dc_dense_backward(ev.ctx, B.DcDenseBackwardArgs(**{**back, **bad})) == want, bad
    off = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    norm = dict(dtype=B.DC_F32, act=0, rows=8, n_graphs=2, channels=8, groups=2, eps=1e-5, node_off=off.data_ptr(), X=x.data_ptr(), ldx=8,
                mean=w.data_ptr(), rstd=w.data_ptr() + 64, Y=y.data_ptr(), ldy=8)
    far = (1 << 17) + 1
    for bad in (dict(ldx=far), dict(ldy=far)):
        assert B.dc_graph_norm(ev.ctx, B.DcGraphNormArgs(**{**norm, **bad})) == B.DC_ERR_UNSUPPORTED, bad
    for bad in (dict(lddy=far), dict(lddx=far), dict(dres=z.data_ptr(), lddres=far)):
        args = {**norm, **dict(dY=z.data_ptr(), lddy=8, dX=y.data_ptr(), lddx=8), **bad}
        assert B.dc_graph_norm_backward(ev.ctx, B.DcGraphNormArgs(**args)) == B.DC_ERR_UNSUPPORTED, bad
    torch.cuda.synchronize()
    assert all((v == 0).all() for v in (x, w, y, z)) and ev.check() == B.DC_OK


def test_c_calls_refuse_results_that_overlap(B, ev):
    """A result in what the call still reads, in another result or in the workspace: refused with nothing enqueued, also where
    the arrays only touch, or begin alike with rows at other distances."""
    n, buf = 16, torch.zeros(40 * 64, device="cuda")
    at = lambda i: buf.data_ptr() + 4 * i
    X, W, Y, Z, R, V, S = (at(i * 256) for i in range(7))                 # arrays of 16 x 16, one behind the other
    ok = dict(dtype=B.DC_F32, act=1, rows=n, n_in=n, n_out=n, X=X, ldx=n, W=W, ldw=n, Y=Y, ldy=n, Z=Z, ldz=n, residual=R, ld_residual=n, bias=V)
    for bad in (dict(Y=R, ldy=n + 4), dict(Y=R + 4 * n), dict(Y=X + 4), dict(Y=X - 4 * n), dict(Y=W), dict(Y=V - 4), dict(Z=W), dict(Z=V),
                dict(Z=R), dict(Z=R - 4, ldz=n), dict(Z=Y + 4 * n), dict(Z=X, ldz=n + 1)):
        assert B.dc_dense(ev.ctx, B.DcDenseArgs(**{**ok, **bad})) == B.DC_ERR_INVALID_ARG, bad
    need = B.dc_dense_backward_bytes(ev.ctx, B.DC_F32, 1, n, n, n)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    kept = B.DcKeptRows(S, S + 1024, 32, 1)
    back = dict(dtype=B.DC_F32, act=1, rows=n, n_in=n, n_out=n, dY=Y, lddy=n, Z=Z, ldz=n, X=X, ldx=n, W=W, ldw=n, dX=R, lddx=n, dW=V, lddw=n,
                db=at(9 * 256), workspace=ws.data_ptr(), workspace_bytes=need)
    for bad in (dict(dX=Y + 4), dict(dX=Z - 4), dict(dX=X + 4 * n), dict(dX=W), dict(dW=Y), dict(dW=Z), dict(dW=X), dict(dW=R + 4), dict(db=Y),
                dict(db=Z), dict(db=X), dict(db=W), dict(db=R + 64), dict(db=V), dict(workspace=X), dict(dX=ws.data_ptr() + need - 16),
                dict(dW=ws.data_ptr()), dict(db=ws.data_ptr() + 64), dict(kept=kept, dX=S + 64), dict(kept=kept, dW=S + 1024 - 16)):
        args = {**back, **{k: v for k, v in bad.items() if k != "kept"}}
        if "kept" in bad:
            args["kept"] = B.C.pointer(bad["kept"])
        assert B.dc_dense_backward(ev.ctx, B.DcDenseBackwardArgs(**args)) == B.DC_ERR_INVALID_ARG, bad
    off = torch.tensor([0, 9, n], dtype=torch.int32, device="cuda")
    norm = dict(dtype=B.DC_F32, act=0, rows=n, n_graphs=2, channels=n, groups=2, eps=1e-5, node_off=off.data_ptr(), X=X, ldx=n, gamma=V, beta=V + 64,
                mean=V + 128, rstd=V + 144, Y=Y, ldy=n)
    for bad in (dict(Y=X, ldy=n + 4), dict(Y=X + 4 * n), dict(Y=V - 4), dict(Y=V + 64), dict(Y=off.data_ptr()), dict(mean=X), dict(rstd=V + 132), dict(mean=Y),
                dict(mean=V), dict(rstd=V + 64), dict(rstd=off.data_ptr() + 4)):
        assert B.dc_graph_norm(ev.ctx, B.DcGraphNormArgs(**{**norm, **bad})) == B.DC_ERR_INVALID_ARG, bad
    need = B.dc_graph_norm_bytes(ev.ctx, n, 2, n, 2, True)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    norm = {**norm, **dict(Y=0, dY=Y, lddy=n, dres=Z, lddres=n, dX=R, lddx=n, dgamma=V + 256, dbeta=V + 320, workspace=ws.data_ptr(), workspace_bytes=need)}
    for bad in (dict(dX=Y, lddx=n + 4), dict(dX=Z, lddx=n + 4), dict(dX=X, lddx=n + 4), dict(dX=Y + 4), dict(dX=Z - 4 * n), dict(dX=V), dict(dX=V + 136),
                dict(dX=off.data_ptr()), dict(dgamma=V + 316), dict(dX=V + 256), dict(workspace=X), dict(dX=ws.data_ptr()), dict(dgamma=ws.data_ptr()),
                dict(kept=kept, dX=S + 64), dict(kept=kept, dX=S + 1024 - 64)):
        args = {**norm, **{k: v for k, v in bad.items() if k != "kept"}}
        if "kept" in bad:
            args["kept"] = B.C.pointer(bad["kept"])
        assert B.dc_graph_norm_backward(ev.ctx, B.DcGraphNormArgs(**args)) == B.DC_ERR_INVALID_ARG, bad
    for x, k in ((S + 64, kept), (S + 1024 - 4, kept), (X, B.DcKeptRows(S, S + 32, 32, 1))):
        assert B.dc_keep_rows(ev.ctx, B.DC_F32, n, n, x, n, k) == B.DC_ERR_INVALID_ARG
    assert B.dc_restore_rows(ev.ctx, B.DC_F32, n, n, kept, S + 64, n) == B.DC_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert not buf.any() and not ws.any() and ev.check() == B.DC_OK
    y = torch.zeros(32, 24, device="cuda")
    with pytest.raises(B.DiscoError):                      # the residual's rows at another distance than those of the result
        ev.dense(torch.ones(16, 8, device="cuda"), torch.ones(8, 16, device="cuda"), residual=y[:16, :16], out=y.view(16, 48)[:, :16])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 300, 5000])
def test_results_beside_what_is_read(ev, dtype, rows):
    """Columns of one matrix as the arrays of a call, each beside the others, and what may be done in place."""
    t, C, G = TYPES[dtype], 32, 4
    big = rand(1, rows, 4 * C).to(t).cuda()
    x, dy, y, z = (big[:, i * C:(i + 1) * C] for i in range(4))
    w, off = (rand(2, C, C) / 6).to(t).cuda(), offsets([rows // 3, rows - rows // 3])
    copies = [v.clone() for v in (x, dy)]
    want = ev.dense(copies[0], w, act="silu")
    ev.dense(x, w, act="silu", out=y)
    assert torch.equal(y, want)
    want, mean, rstd = ev.graph_norm(copies[0], off, G, act="gelu")
    ev.graph_norm(x, off, G, act="gelu", out=z)
    assert torch.equal(z, want) and torch.equal(x, copies[0]) and torch.equal(dy, copies[1])
    want = ev.graph_norm_backward(copies[1], copies[0], off, G, None, None, mean, rstd, "gelu", residual=copies[0])
    for place in (x, dy):                                  # in place of the rows, of the gradient
        keep = place.clone()
        got = ev.graph_norm_backward(dy, x, off, G, None, None, mean, rstd, "gelu", residual=x, out=place)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        place.copy_(keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(700, 96, 139), (33, 40, 70), (8000, 64, 131), (4500, 32, 255)])
def test_dense_adds_to_its_residual_in_place(ev, dtype, shape):
    """Y may be the residual's array; vectors that the columns end in are formed twice and have to find the old values."""
    M, K, N = shape
    x, w, b, r = (rand(i, *s).to(TYPES[dtype]) for i, s in enumerate([(M, K), (K, N), (N,), (M, N)], 11))
    b = b.float()
    want = ev.dense(x.cuda(), w.cuda(), b.cuda(), "silu", r.cuda())
    y = r.cuda()
    ev.dense(x.cuda(), w.cuda(), b.cuda(), "silu", y, out=y)
    assert torch.equal(y, want)


def test_c_calls_refuse(B, ev):
    x = torch.zeros(4, 8, device="cuda")
    ok = dict(dtype=B.DC_F32, act=0, rows=4, n_in=8, n_out=8, X=x.data_ptr(), ldx=8, W=x.data_ptr(), ldw=8, Y=x.data_ptr(), ldy=8)
    for bad, want in [(dict(dtype=3), B.DC_ERR_INVALID_ARG), (dict(act=9), B.DC_ERR_INVALID_ARG), (dict(rows=-1), B.DC_ERR_INVALID_ARG),
                      (dict(rows=1 << 31), B.DC_ERR_UNSUPPORTED), (dict(n_in=0), B.DC_ERR_INVALID_ARG),
                      (dict(n_out=1 << 17), B.DC_ERR_UNSUPPORTED), (dict(X=0), B.DC_ERR_INVALID_ARG), (dict(ldx=7), B.DC_ERR_INVALID_ARG),
                      (dict(W=0), B.DC_ERR_INVALID_ARG), (dict(Y=0), B.DC_ERR_INVALID_ARG), (dict(ldy=3), B.DC_ERR_INVALID_ARG),
                      (dict(X=x.data_ptr() + 2), B.DC_ERR_INVALID_ARG), (dict(residual=x.data_ptr(), ld_residual=2), B.DC_ERR_INVALID_ARG),
                      (dict(bias=x.data_ptr() + 1), B.DC_ERR_INVALID_ARG)]:
        assert B.dc_dense(ev.ctx, B.DcDenseArgs(**{**ok, **bad})) == want, bad
        assert B.dc_last_error(ev.ctx)
    back = dict(dtype=B.DC_F32, act=0, rows=4, n_in=8, n_out=8, dY=x.data_ptr(), lddy=8, X=x.data_ptr(), ldx=8, W=x.data_ptr(), ldw=8,
                dW=x.data_ptr(), lddw=8)
    assert B.dc_dense_backward(ev.ctx, B.DcDenseBackwardArgs(**back)) == B.DC_ERR_CAPACITY
    assert B.dc_dense_backward(ev.ctx, B.DcDenseBackwardArgs(**{**back, "act": 1})) == B.DC_ERR_INVALID_ARG     # no Z
    assert B.dc_dense_backward(ev.ctx, B.DcDenseBackwardArgs(**{**back, "X": 0})) == B.DC_ERR_INVALID_ARG
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    norm = dict(dtype=B.DC_F32, act=0, rows=4, n_graphs=2, channels=8, groups=2, eps=1e-5, node_off=off.data_ptr(), X=x.data_ptr(), ldx=8,
                mean=x.data_ptr(), rstd=x.data_ptr(), Y=x.data_ptr(), ldy=8)
    for bad, want in [(dict(groups=3), B.DC_ERR_INVALID_ARG), (dict(eps=0.0), B.DC_ERR_INVALID_ARG), (dict(node_off=0), B.DC_ERR_INVALID_ARG),
                      (dict(n_graphs=-1), B.DC_ERR_INVALID_ARG), (dict(channels=8200, groups=2), B.DC_ERR_UNSUPPORTED),
                      (dict(channels=2048, groups=1), B.DC_ERR_UNSUPPORTED), (dict(rows=5000), B.DC_ERR_CAPACITY),
                      (dict(mean=0), B.DC_ERR_INVALID_ARG), (dict(ldy=7), B.DC_ERR_INVALID_ARG)]:
        assert B.dc_graph_norm(ev.ctx, B.DcGraphNormArgs(**{**norm, **bad})) == want, bad
    assert B.dc_graph_norm_backward(ev.ctx, B.DcGraphNormArgs(**norm)) == B.DC_ERR_INVALID_ARG                  # no dY
    kept = B.DcKeptRows(x.data_ptr(), x.data_ptr(), 31, 1)
    assert B.dc_keep_rows(ev.ctx, B.DC_F32, 4, 8, x.data_ptr(), 8, kept) == B.DC_ERR_INVALID_ARG
    assert B.dc_keep_rows(ev.ctx, B.DC_F32, 4, 0, x.data_ptr(), 8, B.DcKeptRows(x.data_ptr(), x.data_ptr(), 32, 1)) == B.DC_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert ev.check() == B.DC_OK
