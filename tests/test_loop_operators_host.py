"""Argument checks of the operators for training loops that need no GPU: the binding's own, and the library's where there is no
context."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2209_12769_amd import binding as B


@pytest.fixture()
def ev():
    """An Evaluator without a context, its tensors on the CPU: calls get as far as the library, which refuses them."""
    e = B.Evaluator.__new__(B.Evaluator)
    e.torch, e.device, e.ctx = torch, torch.device("cpu"), None
    e._raw_stream = lambda: 0
    return e


def refused(message, call, *args, **kw):
    with pytest.raises(ValueError, match=message):
        call(*args, **kw)


def without_context(call, *args, **kw):
    with pytest.raises(B.DiscoError) as e:
        call(*args, **kw)
    assert e.value.status == B.DC_ERR_INVALID_ARG


def test_row_norm(ev):
    x, v = torch.zeros(3, 8), torch.zeros(8)
    without_context(ev.row_norm, x, v, v)
    refused("need a matrix", ev.row_norm, torch.zeros(8))
    refused("float32 or bfloat16", ev.row_norm, x.double())
    refused("neighbours", ev.row_norm, torch.zeros(8, 3).t())
    refused("gamma", ev.row_norm, x, torch.zeros(7))
    refused("beta", ev.row_norm, x, v, v.bfloat16())
    refused("unknown activation", ev.row_norm, x, v, v, 1e-5, "tanh")
    refused("out", ev.row_norm, x, v, v, out=torch.zeros(3, 9))
    refused("out", ev.row_norm, x, out=x.bfloat16())
    s = torch.zeros(3)
    without_context(ev.row_norm_backward, x, x, v, v, s, s)
    refused("mean", ev.row_norm_backward, x, x, v, v, torch.zeros(4), s)
    refused("rstd", ev.row_norm_backward, x, x, v, v, s, torch.zeros(3, 1))
    refused("x: need", ev.row_norm_backward, x, torch.zeros(2, 8), v, v, s, s)
    refused("residual", ev.row_norm_backward, x, x, v, v, s, s, residual=x.bfloat16())
    kept = B.KeptRows(torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3, 1, dtype=torch.uint8), 9)
    refused("kept rows", ev.row_norm_backward, x, kept, v, v, s, s)


def test_embed_rows(ev):
    table, ids, dy = torch.zeros(5, 8), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 8)
    without_context(ev.embed_rows, ids, table)
    refused("ids", ev.embed_rows, ids.long(), table)
    refused("ids", ev.embed_rows, ids[None], table)
    refused("ids", ev.embed_rows, torch.zeros(6, dtype=torch.int32)[::2], table)
    refused("table", ev.embed_rows, ids, table.half())
    refused("out", ev.embed_rows, ids, table, out=torch.zeros(4, 8))
    without_context(ev.embed_rows_backward, dy, ids, 5)
    refused("one number for each row", ev.embed_rows_backward, dy, ids[:2], 5)
    refused("out", ev.embed_rows_backward, dy, ids, 5, out=torch.zeros(4, 8))
    refused("kinds", ev.embed_rows_backward, dy, ids, 0)


def test_adamw(ev):
    p, q = torch.zeros(3, 5), torch.zeros(300, dtype=torch.bfloat16)
    o = ev.adamw([p, q], weight_decay=[0.1, 0.0], states="8bit")
    assert o.at == [0, 128] and o.total == 512 and o.m.dtype == torch.uint8 and o.low.numel() == 512 and o.m_exponent.numel() == 4
    assert ev.adamw([p]).low is None and ev.adamw([p]).m.dtype == torch.float32 and ev.adamw([]).total == 0
    refused("states", ev.adamw, [p], states="4bit")
    refused("weight_decay", ev.adamw, [p, q], weight_decay=[0.1])
    refused("tensor 1", ev.adamw, [p, torch.zeros(4, 3).t()])
    refused("tensor 0", ev.adamw, [p.double()])
    refused("2 gradients", o.step, [p])
    refused("which", o.values, "x")
    refused("which", o.values, "ww")
    refused("which", o.values, "")
    without_context(o.values, "w")
    for name in ("m", "v", "low", "steps", "params"):
        with pytest.raises(AttributeError, match="copy_"):
            setattr(o, name, None)
    o.lr = 0.5


def test_adamw_parameters_with_other_memory(ev):
    """Their table follows them; memory that they had cannot become another tensor's before that."""
    p, q = torch.zeros(3, 5), torch.zeros(300, dtype=torch.bfloat16)
    o = ev.adamw([p, q])
    was = q.data_ptr()
    q.data = torch.ones(300, dtype=torch.bfloat16)
    assert torch.zeros(300, dtype=torch.bfloat16).data_ptr() != was and o._table["p"][1] == was
    without_context(o.values, "w")
    assert o._table["p"].tolist() == [p.data_ptr(), q.data_ptr()]
    for other in (torch.zeros(0, dtype=torch.bfloat16), torch.zeros(10, dtype=torch.bfloat16), torch.zeros(300)):
        q.data = other
        refused("tensor 1", o.values, "w")
        refused("tensor 1", o.step, [None, None])


@pytest.mark.parametrize("name,args", [("dc_row_norm", 1), ("dc_row_norm_backward", 1), ("dc_embed_rows", 1), ("dc_embed_rows_backward", 1), ("dc_adamw", 1), ("dc_adamw_values", 4)])
def test_calls_without_a_context(name, args):
    assert getattr(B.lib(), name)(None, *[None] * args, None) == B.DC_ERR_INVALID_ARG


def test_workspaces_without_a_context():
    assert B.dc_row_norm_bytes(None, 5, 8) == 0 and B.dc_embed_rows_bytes(None, 5, 5, 8) == 0


def test_structs_have_the_header_s_layout(tmp_path):
    """Offsets of every field as the C compiler has them."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"dc_row_norm_args": B.DcRowNormArgs, "dc_embed_rows_args": B.DcEmbedRowsArgs, "dc_adamw_args": B.DcAdamwArgs, "dc_adamw_tensor": B.DcAdamwTensor}
    lines = ['printf("%%zu", sizeof(%s));' % s + "".join('printf(" %%zu", offsetof(%s, %s));' % (s, f[0]) for f in c._fields_) + 'printf("\\n");' for s, c in structs.items()]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "disco.h"\nint main(void) { %s return 0; }\n' % "\n".join(lines))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", str(tmp_path / "layout"), str(src)], check=True)
    got = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines()
    for line, c in zip(got, structs.values()):
        assert list(map(int, line.split())) == [ctypes.sizeof(c)] + [getattr(c, f[0]).offset for f in c._fields_]
    assert np.dtype(B._ADAMW_TENSOR).itemsize == ctypes.sizeof(B.DcAdamwTensor)


def test_adamw_looks_at_every_gradient(ev):
    """What the table holds of gradients, some of them missing, of types that change from step to step."""
    ps = [torch.zeros(3, 5), torch.zeros(7), torch.zeros(0), torch.zeros(300, dtype=torch.bfloat16)]
    o = ev.adamw(ps)
    good = [torch.zeros_like(p) for p in ps]
    half = [g.bfloat16() for g in good]
    for grads in (good, [None, good[1], None, good[3]], half, good, [half[0], None, half[2], None], [None] * 4, tuple(half), good):
        without_context(o.step, grads)
        assert o._table["g"].tolist() == [0 if g is None else g.data_ptr() for g in grads]
        assert all(g is None or code == (g.dtype == torch.bfloat16) for g, code in zip(grads, o._table["g_dtype"].tolist()))
    for k, bad in [(0, torch.zeros(5, 3)), (0, torch.zeros(5, 3).t()), (1, torch.zeros(7).double()), (1, torch.zeros(1).expand(7)), (3, torch.zeros(299)),
                   (2, torch.zeros(1))]:
        for rest in (good, [None] * 4):
            refused(f"gradient {k}", o.step, [bad if i == k else g for i, g in enumerate(rest)])


def test_adamw_looks_at_the_layout_of_parameters(ev):
    """A parameter whose order, type or shape changed while its memory is the same: refused, and taken again once it is as it was."""
    def changed(p):
        yield "transposed", lambda: p.t_(), lambda: p.t_()
        was = p.data
        for name, other in [("transposed data", was.t()), ("overlapping rows", was.as_strided((16, 16), (8, 1))), ("another type", was.flatten().view(torch.bfloat16)[:256].view(16, 16)),
                            ("no type of a parameter", was.view(torch.int32)), ("fewer rows", was[:9]), ("another shape", was.view(8, 32)), ("a vector", was.view(256))]:
            assert other.data_ptr() == was.data_ptr()
            yield name, lambda: setattr(p, "data", other), lambda: setattr(p, "data", was)
    params = [torch.zeros(7), torch.arange(256.0).view(16, 16)]
    o = ev.adamw(params)
    grads = [torch.zeros_like(p) for p in params]
    without_context(o.step, grads)
    for name, change, undo in changed(params[1]):
        change()
        for call, args in ((o.step, [grads]), (o.step, [[None, grads[1]]]), (o.values, ["w"])):
            try:
                refused("tensor 1", call, *args)
            except B.DiscoError:
                pytest.fail(f"{name}: {call.__name__} went on to the library")
        undo()
        without_context(o.step, grads)
        without_context(o.values, "w")


def test_adamw_has_the_parameters_that_it_was_made_of(ev):
    """The list of them is no place to add or to take away any."""
    params = [torch.zeros(7), torch.zeros(7)]
    for change in (lambda ps: ps.append(torch.zeros(7)), lambda ps: ps.pop(), lambda ps: ps.pop(0)):
        o = ev.adamw(params)
        change(o.params)
        refused("2 tensors", o.step, [torch.zeros(7)] * 2)
        refused("2 gradients", o.step, [torch.zeros(7)] * len(o.params))
        refused("2 tensors", o.values, "w")


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_adamw_state_given_other_memory(ev, states):
    """The calls go by where the state lies: a part of it that has other memory, or none, is refused, and what it had is not
    another tensor's while the calls would write there."""
    q = torch.zeros(300, dtype=torch.bfloat16)
    o = ev.adamw([q], states=states)
    for name in ["m", "v", "low", "steps"] + (["m_exponent", "v_exponent"] if states == "8bit" else []):
        part = getattr(o, name)
        was, memory = part.data_ptr(), part.data
        for other in (part.clone(), part.data[1:], torch.zeros(0, dtype=part.dtype)):
            part.data = other
            refused(name, o.step, [q.clone()])
            refused(name, o.values, "w")
        del memory
        taken = [torch.zeros_like(part) for _ in range(20)] + [torch.zeros(n, dtype=part.dtype) for n in (2, 4, 384, 768)]
        assert all(t.data_ptr() != was for t in taken), name
        o = ev.adamw([q], states=states)
    without_context(o.step, [q.clone()])
