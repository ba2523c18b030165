"""Norms and rotations of Q and K on the host: the table against the oracle, and what the entry points refuse before anything is
launched (CPU only: addresses here are never read)."""
import ctypes

import numpy as np
import pytest

from oracle import paro_norm_rope as on
from paper_2506_16054_amd import binding as pb


def at(i, offset=0):
    return (i + 1) * (1 << 30) + offset


@pytest.mark.parametrize("grid,dims,d", [((1, 1, 1), (16, 24, 24), 64), ((3, 4, 5), (20, 22, 22), 64), ((2, 3, 2), (0, 64, 64), 128),
                                         ((2, 1, 3), (0, 0, 2), 64), ((2, 2, 2), (0, 0, 0), 64)])
def test_table_is_the_oracles(grid, dims, d):
    s, axes = pb.make_shape(1, 1, d, *grid, 5, 64), pb.make_rope_axes(dims)
    rng = np.random.default_rng(3)
    pos = [rng.uniform(-1e5, 1e5, n) for n in grid]
    freq = [rng.uniform(0, 1, k // 2) for k in dims]
    assert pb.paro_rope_table_floats(s, axes) == sum(n * k for n, k in zip(grid, dims))
    got = pb.paro_rope_table(s, axes, pos, freq)
    want = on.rope_table(grid, dims, np.concatenate(pos), np.concatenate(freq))
    assert got.dtype == np.float32 and got.shape == want.shape
    # the two binary64 functions may differ in their last bit, and the rounding to float32 with them
    assert np.all(np.abs(got - want) <= 2.0**-23 * np.abs(want))
    assert np.mean(got == want) >= 0.99 if got.size else True
    assert np.array_equal(pb.paro_rope_table(s, axes, np.concatenate(pos), np.concatenate(freq)), got)


def test_table_refusals():
    s = pb.make_shape(1, 1, 64, 2, 3, 4, 0, 64)
    for axes in (pb.make_rope_axes((15, 24, 24)), pb.make_rope_axes((-2, 24, 24)), pb.make_rope_axes((16, 24, 26)), pb.make_rope_axes((16, 24, 24), 2)):
        with pytest.raises(pb.ParoError) as e:
            pb.paro_rope_table_floats(s, axes)
        assert e.value.status == pb.PARO_EINVAL
    axes = pb.make_rope_axes((16, 24, 24))
    with pytest.raises(pb.ParoError):
        pb.paro_rope_table(s, axes, np.zeros(8), np.zeros(32))
    with pytest.raises(pb.ParoError):
        pb.paro_rope_table(s, axes, np.zeros(9), np.zeros(31))
    L = pb.lib()
    assert L.paro_rope_table_floats(None, ctypes.byref(axes)) == pb.PARO_EINVAL and L.paro_rope_table_floats(ctypes.byref(s), None) == pb.PARO_EINVAL
    assert L.paro_rope_table(ctypes.byref(s), ctypes.byref(axes), None, None, None) == pb.PARO_EINVAL


class Call:
    """The arguments of the four entry points, all valid, as addresses that nothing reads; `change` makes one of them invalid."""
    N = 2 * 3 * 4 + 5

    def __init__(self):
        d, nh, n = 64, 3, self.N
        self.s = pb.make_shape(2, nh, d, 2, 3, 4, 5, 64)
        self.axes = pb.make_rope_axes((16, 24, 24))
        self.dtype, self.table, self.bits, self.ids = pb.PARO_BF16, at(50), (8, 8), (ctypes.c_uint8 * 3)(0, 3, 5)
        self.norm = pb.paro_qk_norm(kind=pb.PARO_NORM_LAYER, eps=1e-6)
        self.rows = [pb.paro_strided(at(i), nh * n * d, n * d, d) for i in range(6)]
        self.grad = pb.paro_qk_norm_grad()
        for i in range(2):
            self.norm.weight[i], self.norm.bias[i] = at(20 + i), at(22 + i)
            self.grad.weight[i], self.grad.bias[i] = at(24 + i), at(26 + i)
        self.scratch, self.codes, self.scales = at(30), [at(31 + i) for i in range(3)], [at(34 + i) for i in range(3)]

    def refused(self, which):
        L, b = pb.lib(), ctypes.byref
        r = [None if x is None else b(x) for x in self.rows]
        s, axes, norm = (None if x is None else b(x) for x in (self.s, self.axes, self.norm))
        if which == "rope":
            st = L.paro_rope(s, self.dtype, axes, self.table, 0, r[0], r[1], None)
        elif which == "forward":
            st = L.paro_qk_norm_rope(s, self.dtype, axes, self.table, norm, *r[:4], None)
        elif which == "backward":
            st = L.paro_qk_norm_rope_backward(s, self.dtype, axes, self.table, norm, *r, None if self.grad is None else b(self.grad), self.scratch, None)
        else:
            c, f = self.codes, self.scales
            st = L.paro_qk_norm_rope_quantize_qkv(s, self.dtype, *self.bits, self.ids, axes, self.table, norm, *r[:3], c[0], f[0], c[1], f[1], c[2], f[2],
                                                  None)
        assert st in (pb.PARO_EINVAL, pb.PARO_EUNSUPPORTED), st
        assert L.paro_last_error()
        return True


ALL = ("rope", "forward", "backward", "quantize")


def _set(path, value):
    def change(c):
        *head, last = path
        for p in head:
            c = c[p] if isinstance(p, int) else getattr(c, p)
        if isinstance(last, int):
            c[last] = value
        else:
            setattr(c, last, value)
    return change


COMMON = {
    "no shape": _set(("s",), None), "a shape of no heads": _set(("s", "nh"), 0), "another head dimension": _set(("s", "d"), 96), "no axes": _set(("axes",), None),
    "odd channels": _set(("axes", "dims", 0), 15), "more channels than a row": _set(("axes", "dims", 2), 26), "no way to pair": _set(("axes", "pairs"), 7),
    "a type": _set(("dtype",), 2), "no table": _set(("table",), None), "a table off its bytes": _set(("table",), at(50, 8)),
    "no input": _set(("rows", 0), None), "an input's null": _set(("rows", 0, "data"), None), "an input off its bytes": _set(("rows", 0, "data"), at(0, 8)),
    "a negative stride": _set(("rows", 0, "token"), -64), "a stride off its bytes": _set(("rows", 0, "token"), 68), "a stride beyond all memory": _set(("rows", 0, "batch"), 1 << 60), "a token stride of 2^31": _set(("rows", 0, "token"), 1 << 31),
}


@pytest.mark.parametrize("which", ALL)
@pytest.mark.parametrize("what", sorted(COMMON))
def test_common_refusals(which, what):
    c = Call()
    COMMON[what](c)
    assert c.refused(which)


OUTPUTS = {"no output": lambda r: setattr(r, "data", None), "rows on each other": lambda r: setattr(r, "token", 32), "one row for all tokens": lambda r: setattr(r, "token", 0),
           "heads on each other": lambda r: setattr(r, "head", 64), "batches on each other": lambda r: setattr(r, "batch", 64),
           "a batch inside a head": lambda r: setattr(r, "batch", 64 * Call.N)}


@pytest.mark.parametrize("which,first,last", [("rope", 1, 2), ("forward", 2, 4), ("backward", 4, 6)])
@pytest.mark.parametrize("what", sorted(OUTPUTS))
def test_refused_outputs(which, first, last, what):
    for i in range(first, last):
        c = Call()
        OUTPUTS[what](c.rows[i])
        assert c.refused(which)


@pytest.mark.parametrize("which,outs,ins", [("rope", (1,), (0,)), ("forward", (2, 3), (0, 1)), ("backward", (4, 5), (0, 1, 2, 3))])
def test_outputs_in_the_memory_of_others(which, outs, ins):
    for o in outs:
        for i in ins + outs:
            if i == o:
                continue
            c = Call()
            c.rows[o].data = c.rows[i].data
            if i % 2 == o % 2 or which == "rope":  # its own input: refused in another order only
                c.rows[o].head, c.rows[o].token = 64, 3 * 64
                c.rows[o].batch = 3 * 64 * Call.N
            assert c.refused(which)


NORMS = {
    "no norm": _set(("norm",), None), "a kind": _set(("norm", "kind"), 3), "a negative eps": _set(("norm", "eps"), -1e-6), "an eps that is no number": _set(("norm", "eps"), float("nan")),
    "an infinite eps": _set(("norm", "eps"), float("inf")), "weights without a norm": _set(("norm", "kind"), 0), "biases of a root mean square": _set(("norm", "kind"), 1),
    "a weight off its bytes": _set(("norm", "weight", 1), at(20, 4)), "a text bias off its bytes": _set(("norm", "text_bias", 0), at(20, 8)),
}


@pytest.mark.parametrize("which", ALL[1:])
@pytest.mark.parametrize("what", sorted(NORMS))
def test_refused_norms(which, what):
    c = Call()
    NORMS[what](c)
    assert c.refused(which)


GRADS = {
    "a gradient off its bytes": _set(("grad", "weight", 0), at(24, 4)), "two in one place": _set(("grad", "bias", 0), at(24)),
    "of text weights that are not there": _set(("grad", "text_weight", 0), at(40)), "of text biases that are not there": _set(("grad", "text_bias", 1), at(40)),
    "no scratch": _set(("scratch",), None), "scratch off its bytes": _set(("scratch",), at(30, 8)),
}


@pytest.mark.parametrize("what", sorted(GRADS))
def test_refused_gradients(what):
    c = Call()
    GRADS[what](c)
    assert c.refused("backward")


def test_gradients_of_what_the_norm_has_not():
    c = Call()
    c.norm = pb.paro_qk_norm(kind=pb.PARO_NORM_NONE)
    assert c.refused("backward")
    c.norm = pb.paro_qk_norm(kind=pb.PARO_NORM_RMS, eps=1e-6)
    assert c.refused("backward")


QUANT = {
    "bits": _set(("bits",), (8, 16)), "no order ids": _set(("ids",), None), "an order id": _set(("ids", 1), 6), "no codes": _set(("codes", 1), None),
    "no scales": _set(("scales", 2), None), "codes off their bytes": _set(("codes", 0), at(31, 8)), "codes in an input": _set(("codes", 2), at(0)),
    "codes twice": _set(("codes", 2), at(31)), "scales twice": _set(("scales", 2), at(34)), "no v": _set(("rows", 2), None),
}


@pytest.mark.parametrize("what", sorted(QUANT))
def test_refused_quantizers(what):
    c = Call()
    QUANT[what](c)
    assert c.refused("quantize")


def test_scratch_bytes():
    assert pb.paro_qk_norm_rope_backward_bytes(pb.make_shape(1, 1, 64, 1, 1, 1, 0, 64)) > 0
    with pytest.raises(pb.ParoError):
        pb.paro_qk_norm_rope_backward_bytes(pb.make_shape(1, 1, 48, 1, 1, 1, 0, 64))


def test_binding_refuses_host_tensors_and_unknown_vectors():
    import torch

    s, axes = pb.make_shape(1, 1, 64, 1, 1, 1, 0, 64), pb.make_rope_axes((16, 24, 24))
    x = torch.zeros((1, 1, 1, 64))
    with pytest.raises(pb.ParoError):
        pb.paro_rope(s, axes, torch.zeros((32, 2)), x, x)
    with pytest.raises(pb.ParoError, match="qweight"):
        pb.QkNorm(pb.PARO_NORM_RMS, 1e-6, qweight=x)
    with pytest.raises(pb.ParoError):
        pb.paro_qk_norm_rope(s, axes, None, pb.QkNorm(pb.PARO_NORM_NONE), x, x, x, x)


def test_tensors_of_another_device_are_refused():
    """On a machine with one GPU the second device is a stand-in that answers as its tensors would."""
    import types

    far = types.SimpleNamespace(is_cuda=True, shape=(1, 1, 1, 64), dtype="bf16", stride=lambda i=None: 1 if i == 3 else (64, 64, 64, 1),
                                get_device=lambda: 1, data_ptr=lambda: at(0))
    with pytest.raises(pb.ParoError, match="device 1"):
        pb._strided(far, "x", (1, 1, 1, 64), "bf16", 0)
    assert pb._strided(far, "x", (1, 1, 1, 64), "bf16", 1).data == at(0)
