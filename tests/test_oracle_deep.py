"""The oracle of deep estimators against closed forms and differences, and the refusals of the operators' binding (no GPU)."""
import numpy as np
import pytest

from oracle import deep
from oracle import oracle as orc
from oracle import train as ot
from paper_2209_12769_amd import binding as B
from paper_2209_12769_amd import workloads as wl


def small(L=3, H=32, seed=3):
    g = wl.random_dag(seed, 14, 0.2, 16)
    w = wl.custom("deep", wl.ModelSpec(16, H, L, "f32"), [g], [wl.random_labels(seed, 14, 6, 3)], seed=seed, std=0.2)
    w.weights.head[-H - 1:-1] = np.abs(w.weights.head[-H - 1:-1])       # estimates above the floor: it has no gradient below
    w.weights.head[-1] += 3.0
    b = orc.contract(w)
    rng = np.random.default_rng(seed)
    p = ot.Params.from_weights(w.weights, 16, H, L)
    return b, p, 1 + 0.2 * rng.standard_normal((L - 1, H)), 0.2 * rng.standard_normal((L - 1, H)), rng.uniform(0.5, 2, b.n_cand)


def test_norm_closed_forms():
    h = np.array([[1.0, 3.0, 5.0, 5.0], [3.0, 1.0, 5.0, 5.0], [7.0, 9.0, 0.0, 2.0]])
    u, xh, r = deep.norm(h, [0, 2, 2, 3], 2, np.ones(4), np.zeros(4), 1e-12, "none")
    assert np.allclose(u, [[-1, 1, 0, 0], [1, -1, 0, 0], [-1, 1, -1, 1]], atol=1e-9)
    assert np.allclose(r[0, :2], 1.0) and np.allclose(r[2], 1.0)


def test_keep_closed_forms():
    x = np.zeros((3, 40))
    x[0, :3] = [127.0, 0.4, -0.2]        # step 1: 0.4 and -0.2 keep their signs
    x[1, 0] = 127.5                      # one step more than 127 of size 1: size 2
    x[1, 39] = 1.0                       # the second block has an exponent of its own: 127 steps of 2^-6 reach 1
    k = deep.keep(x)
    assert list(k[0, :3]) == [127.0, 1.0, -1.0] and k[1, 0] == 128.0 and k[1, 39] == 1.0 and not k[2].any()


@pytest.mark.parametrize("name", deep.ACTS)
def test_gradients_against_differences(name):
    b, p, gamma, beta, t = small()
    loss, y, g, dgamma, dbeta = deep.loss_and_gradients(b, t, p, gamma, beta, 4, 1e-3, name)
    assert (y > 1.0).all() and np.abs(dgamma).max() > 0
    rng = np.random.default_rng(1)

    def value(flat, ga, be):
        y, _ = deep.forward(b, ot.Params.from_flat(flat, 16, 32, 3), ga, be, 4, 1e-3, name)
        return ot.loss_of(y, t, 1e-6)
    flat, o, h = p.flat(), 0, 1e-6
    assert abs(value(flat, gamma, beta) - loss) < 1e-12
    gf = g.flat()
    for shp in ot.Params.shapes(16, 32, 3):
        n = int(np.prod(shp))
        d = np.zeros_like(flat)
        d[o:o + n] = rng.standard_normal(n) / np.sqrt(n)
        num = (value(flat + h * d, gamma, beta) - value(flat - h * d, gamma, beta)) / (2 * h)
        assert abs(num - gf @ d) <= 1e-6 * max(1.0, np.abs(gf[o:o + n]).max()), shp
        o += n
    for which, grad in ((0, dgamma), (1, dbeta)):
        d = rng.standard_normal(gamma.shape) / 8
        s = [(gamma + k * d, beta) if which == 0 else (gamma, beta + k * d) for k in (h, -h)]
        num = (value(flat, *s[0]) - value(flat, *s[1])) / (2 * h)
        assert abs(num - (grad * d).sum()) <= 1e-6 * max(1.0, np.abs(grad).max())


def test_kept_gradient_is_the_gradient_at_kept_values():
    """Values that 8 bits hold exactly give the same gradient; others one that is close."""
    b, p, gamma, beta, t = small()
    plain = deep.loss_and_gradients(b, t, p, gamma, beta, 4, 1e-3, "silu")[2].flat()
    kept = deep.loss_and_gradients(b, t, p, gamma, beta, 4, 1e-3, "silu", kept=True)[2].flat()
    assert 0 < np.linalg.norm(plain - kept) <= 0.05 * np.linalg.norm(plain)


# ---- the binding's own checks, without a device ----
class _NoDevice(B.Evaluator):
    def __init__(self):
        import torch
        self.torch, self.device, self.ctx = torch, torch.device("cpu"), None

    def _stream(self):
        raise AssertionError("a refused call reached the library")


def test_binding_refuses():
    import torch
    ev = _NoDevice()
    x, w, f = torch.zeros(4, 8), torch.zeros(8, 6), torch.float64
    bad = [lambda: ev.dense(x, torch.zeros(7, 6)), lambda: ev.dense(x.to(f), w.to(f)), lambda: ev.dense(x, w.bfloat16()),
           lambda: ev.dense(x.t(), torch.zeros(4, 6)), lambda: ev.dense(x, w, act="tanh"), lambda: ev.dense(x, w, bias=torch.zeros(5)),
           lambda: ev.dense(x, w, residual=torch.zeros(4, 5)), lambda: ev.dense(x, w, out=torch.zeros(3, 6)), lambda: ev.dense(x[0], w),
           lambda: ev.dense_backward(torch.zeros(4, 6), x, w, "silu"), lambda: ev.dense_backward(torch.zeros(5, 6), x, w),
           lambda: ev.dense_backward(torch.zeros(4, 6), B.KeptRows(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 9), w),
           lambda: ev.restore_rows(B.KeptRows(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 8), f),
           lambda: B.KeptRows(torch.zeros(4, 31, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 8),
           lambda: B.KeptRows(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 33),
           lambda: ev.keep_rows(torch.zeros(4, 8, device="meta"))]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", k)


def test_kept_rows_as_a_struct():
    import torch
    code, exponent = torch.zeros(5, 96, dtype=torch.int8), torch.zeros(5, 2, dtype=torch.uint8)
    for k, want in ((B.KeptRows(code[:, :64], exponent, 33), (96, 2)), (B.KeptRows(code[:1].as_strided((1, 64), (7, 1)), exponent[:1], 64), (64, 2))):
        assert (k.c.code, k.c.exponent, k.c.ld_code, k.c.ld_exponent) == (code.data_ptr(), exponent.data_ptr(), *want)


def test_null_contexts_are_errors():
    lib = B.lib()
    for name, args in (("dc_dense", (None, None, None)), ("dc_dense_backward", (None, None, None)), ("dc_graph_norm", (None, None, None)),
                       ("dc_graph_norm_backward", (None, None, None)), ("dc_keep_rows", (None, 0, 0, 1, None, 0, None, None)),
                       ("dc_restore_rows", (None, 0, 0, 1, None, None, 0, None)), ("dc_set_layer_norms", (None, 0, 0, 1e-5, None, None, None)),
                       ("dc_get_layer_norms", (None, None, None, None)), ("dc_train_keep", (None, 0))):
        assert getattr(lib, name)(*args) == B.DC_ERR_INVALID_ARG, name
    assert B.dc_dense_backward_bytes(None, 0, 0, 4, 4, 4) == 0 and B.dc_graph_norm_bytes(None, 4, 1, 4, 1, False) == 0
