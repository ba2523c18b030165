"""Norms of Q and K, their rotation by position, the gradients of both and both with the quantizer, against the float64 oracle.

Tolerances.  Forward values are binary64 rounded to binary32 and, for bf16 outputs, once more: half a step of the output type, plus
half a binary32 step, relative to the value, and 2^-45 of the row's largest term for the binary64 sums themselves.  Codes and scales are
bit for bit those of the separate calls.  Gradients are binary32 arithmetic on a binary64 norm; the bounds count its roundings:
_dx_bound and _dw_bound."""
import numpy as np
import pytest

from oracle import paro_norm_rope as on
from oracle import paro_oracle as po

pytestmark = pytest.mark.gpu

U32 = 2.0**-24


def _pb():
    from paper_2506_16054_amd import binding as pb

    return pb


@pytest.fixture(params=["native", "ctypes"], autouse=True)
def route(request, monkeypatch):
    """Every call through the native module, which must take it, and through the binding's own checks and ctypes."""
    pb = _pb()
    monkeypatch.setattr(pb, "_fast", pb._native() if request.param == "native" else pb._NoNative)
    return request.param


class Problem:
    """Inputs on the device in some memory layout, and the same values in float64 on the host."""

    def __init__(self, B=2, nh=3, d=64, grid=(2, 3, 5), T=0, dims=None, halves=0, dtype="bfloat16", kind="rms", layout="heads", text_norm=False, seed=0,
                 block=64, eps=1e-6, ones=False, start=0.0):
        import torch

        pb = _pb()
        self.B, self.nh, self.d, self.grid, self.T, self.halves, self.kind, self.eps, self.layout = B, nh, d, grid, T, halves, kind, eps, layout
        self.dims = dims = dims or ((16, 24, 24) if d == 64 else (16, 56, 56))
        self.n_img, self.n = int(np.prod(grid)), int(np.prod(grid)) + T
        self.dtype = getattr(torch, dtype)
        self.s = pb.make_shape(B, nh, d, *grid, T, block)
        self.axes = pb.make_rope_axes(dims, pb.PARO_PAIRS_HALVES if halves else pb.PARO_PAIRS_ADJACENT)
        pos = [start + np.arange(x, dtype=np.float64) for x in grid]
        freq = [10000.0 ** (-np.arange(0, x, 2, dtype=np.float64) / x) if x else np.empty(0) for x in dims]
        h_table = pb.paro_rope_table(self.s, self.axes, pos, freq)
        self.table = torch.from_numpy(h_table).to("cuda:0")
        self.cos, self.sin = on.token_angles(grid, T, d, dims, h_table)
        self.gen = torch.Generator().manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        self.x = self.rows(3)
        vectors = {}
        names = [] if kind == "none" or ones else ["weight"] + (["bias"] if kind == "layer" else [])
        for text in ("", "text_") if text_norm else ("",):
            for name in names:
                for x in "qk":
                    vectors[text + x + "_" + name] = (float(name == "weight") + 0.3 * torch.randn((d,), generator=self.gen)).to("cuda:0")
        self.vectors = vectors
        self.norm = pb.QkNorm({"none": pb.PARO_NORM_NONE, "rms": pb.PARO_NORM_RMS, "layer": pb.PARO_NORM_LAYER}[kind], eps, **vectors)

    def empty(self, count=3, fill=None):
        """`count` tensors [B, nh, N, d] in the problem's layout, of values that no call leaves there."""
        import torch

        B, n, nh, d = self.B, self.n, self.nh, self.d
        z = dict(dtype=self.dtype, device="cuda:0")
        if self.layout == "fused":
            self.whole = torch.full((B, n, 3, nh, d), 7.0 if fill is None else fill, **z)
            return list(self.whole.permute(2, 0, 3, 1, 4)[:count])
        if self.layout == "tokens":
            return [torch.full((B, n, nh, d), 7.0, **z).transpose(1, 2) for _ in range(count)]
        return [torch.full((B, nh, n, d), 7.0, **z) for _ in range(count)]

    def rows(self, count):
        import torch

        out = self.empty(count)
        for t in out:
            t.copy_(torch.randn(t.shape, generator=self.gen) * torch.exp(0.5 * torch.randn((self.B, 1, self.n, 1), generator=self.gen)) + 0.25)
        return out

    def w(self, which, name, fallback):
        get = lambda key: None if key not in self.vectors else self.vectors[key].cpu().numpy()
        shared = get(which + "_" + name)
        return on.per_token(np.full(self.d, fallback) if shared is None else shared, get("text_" + which + "_" + name), self.n_img, self.n)

    def forward(self, i):
        which = "qk"[i]
        return on.norm_rope(host(self.x[i]), self.kind, self.eps, self.w(which, "weight", 1.0), self.w(which, "bias", 0.0), self.cos, self.sin, self.halves)


def host(t):
    return t.detach().to("cpu").double().numpy()


def half_step(dtype):
    import torch

    return torch.finfo(dtype).eps / 2


def check_values(got, want, dtype, what):
    """One rounding to binary32, one to the output type; the sums behind a value are as large as its row's largest term."""
    step = half_step(dtype) + (U32 if half_step(dtype) > U32 else 0.0)
    bound = step * (1 + 1e-6) * np.abs(want) + 2.0**-45 * np.abs(want).max(-1, keepdims=True) + 1e-37
    off = np.abs(host(got) - want)
    assert np.all(off <= bound), (what, float((off / bound).max()))


CASES = [
    dict(),
    dict(dtype="float32", kind="layer"),
    dict(dtype="float32", d=128, kind="rms", halves=1, dims=(44, 42, 42)),
    dict(d=128, kind="layer", T=7, text_norm=True, halves=0),
    dict(kind="rms", T=7, text_norm=True, halves=1, layout="fused"),
    dict(kind="none", layout="fused", T=1),
    dict(kind="layer", layout="tokens", dims=(20, 22, 22), halves=1, dtype="float32"),
    dict(kind="rms", dims=(8, 10, 4), halves=0, layout="fused", dtype="float32"),   # channels that do not turn
    dict(kind="rms", dims=(8, 10, 4), halves=1, d=128),
    dict(kind="layer", dims=(0, 0, 0), T=3),                                          # nothing turns
    dict(kind="rms", dims=(0, 64, 64), d=128, grid=(1, 9, 7), layout="tokens"),
    dict(B=1, nh=1, grid=(1, 1, 1), kind="layer", d=64),                              # one token
    dict(B=1, nh=24, grid=(1, 1, 1), kind="rms", d=128, layout="fused", start=977.0),
    dict(B=3, nh=5, grid=(1, 1, 67), kind="rms", T=65, text_norm=True),               # one token more than a tile, of both kinds
    dict(B=1, nh=2, grid=(5, 1, 13), kind="layer", d=128, T=33, text_norm=True, dtype="float32"),
    dict(B=1, nh=48, grid=(3, 11, 13), kind="layer", layout="fused", start=30000.0),
    dict(kind="rms", ones=True), dict(kind="layer", ones=True, dtype="float32"),      # no weights
    dict(kind="rms", eps=10.0),
]


def _id(c):
    return "-".join("%s=%s" % kv for kv in sorted(c.items())) or "plain"


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_rope(case, inverse):
    p = Problem(**case)
    out = p.empty(1)[0]
    _pb().paro_rope(p.s, p.axes, p.table, p.x[0], out, inverse)
    check_values(out, on.turn(host(p.x[0]), p.cos, p.sin, p.halves, inverse), p.dtype, "rope")
    _pb().paro_rope(p.s, p.axes, p.table, p.x[0], p.x[0], inverse)  # in place
    assert np.array_equal(host(p.x[0]), host(out))


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_norm_rope(case):
    p = Problem(**case)
    want = [p.forward(i) for i in range(2)]
    out = p.empty(2)
    _pb().paro_qk_norm_rope(p.s, p.axes, p.table, p.norm, p.x[0], p.x[1], *out)
    for i in range(2):
        check_values(out[i], want[i], p.dtype, "qk"[i])
    if p.layout == "fused":  # the slice that is not an output is left as it was
        assert bool((p.whole[:, :, 2] == 7).all())
    _pb().paro_qk_norm_rope(p.s, p.axes, p.table, p.norm, p.x[0], p.x[1], p.x[0], p.x[1])  # in place
    for i in range(2):
        assert np.array_equal(host(p.x[i]), host(out[i]))


def _abs_turn(x, p):
    """|a c| + |b s| and |a s| + |b c| of every pair: what a turned value's rounding errors scale with."""
    a, b = on.pair_channels(p.d, p.halves)
    y, x, c, s = np.array(np.abs(x)), np.abs(x), np.abs(p.cos), np.abs(p.sin)
    y[..., a], y[..., b] = x[..., a] * c + x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def _bounds(p, which, x, dy):
    """dx = r (g w - m1 - h m2) in binary32: g from one product and one fma (2 roundings of its terms A), g w one more, h one, the two
    means sums of d terms, 8 in a lane, at most 4 steps across lanes and the factor 1/d: 13 roundings each, of terms v (3 roundings) or v h
    (5); then h m2, the differences, the factor r: 4.  28 roundings of the terms' absolute values cover each part.  A weight's
    gradient adds g h (4 roundings) over the heads of a workgroup (at most nh) in binary32, the rest in binary64 with two roundings to
    binary32 on the way."""
    A, w = _abs_turn(dy, p), np.abs(p.w(which, "weight", 1.0))
    if p.kind == "none":
        return 3 * U32 * A, None, None
    h, r = on.normed(x, p.kind, p.eps)
    v, h = A * w, np.abs(h)
    terms = v + h * (v * h).mean(-1, keepdims=True) + (v.mean(-1, keepdims=True) if p.kind == "layer" else 0)
    return 28 * U32 * r * terms, (8 + p.nh) * U32 * A * h, (8 + p.nh) * U32 * A


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_backward(case):
    import torch

    pb = _pb()
    p = Problem(**case)
    dy = p.rows(2)
    dx = p.empty(2)
    grads = {name: torch.full((p.d,), 5.0, device="cuda:0") for name in (p.vectors if p.vectors or p.kind == "none" else ("q_weight", "k_weight"))}
    scratch = torch.full((pb.paro_qk_norm_rope_backward_bytes(p.s),), 255, dtype=torch.uint8, device="cuda:0")  # NaN wherever it is read unwritten
    pb.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm, p.x[0], p.x[1], *dy, *dx, pb.QkNormGrad(**grads), scratch)
    if p.layout == "fused":  # the slice that is not an output is left as it was
        assert bool((p.whole[:, :, 2] == 7).all())
    spans = {"": slice(0, p.n_img), "text_": slice(p.n_img, None)}
    for i, which in enumerate("qk"):
        x, g = host(p.x[i]), host(dy[i])
        want, dw, db = on.norm_rope_backward(x, g, p.kind, p.eps, p.w(which, "weight", 1.0), p.cos, p.sin, p.halves)
        bx, bw, bb = _bounds(p, which, x, g)
        bound = bx + half_step(p.dtype) * (np.abs(want) + bx) + 1e-37
        off = np.abs(host(dx[i]) - want)
        assert np.all(off <= bound), (which, float((off / bound).max()))
        for text, span in spans.items():
            for name, terms, terms_bound in (("weight", dw, bw), ("bias", db, bb)):
                key = text + which + "_" + name
                if key not in grads:
                    continue
                rows = span if "text_" + which + "_" + name in grads else slice(None)
                ref, bound = terms[:, :, rows].sum((0, 1, 2)), terms_bound[:, :, rows].sum((0, 1, 2)) + 1e-37
                off = np.abs(host(grads[key]) - ref)
                assert np.all(off <= bound), (key, float((off / bound).max()))
    # without the norms' gradients, and in the place of the outputs' gradients: the same values
    pb.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm, p.x[0], p.x[1], *dy, *dy)
    for i in range(2):
        assert torch.equal(dy[i], dx[i])


def test_backward_is_the_same_in_every_call():
    import torch

    pb = _pb()
    p = Problem(B=2, nh=7, grid=(5, 17, 23), kind="layer", dtype="float32", T=19, text_norm=True)
    dy = p.rows(2)
    seen = []
    for fill in (0, 255):
        dx, grads = p.empty(2), {name: torch.empty((p.d,), device="cuda:0") for name in p.vectors}
        scratch = torch.full((pb.paro_qk_norm_rope_backward_bytes(p.s),), fill, dtype=torch.uint8, device="cuda:0")
        pb.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm, p.x[0], p.x[1], *dy, *dx, pb.QkNormGrad(**grads), scratch)
        seen.append([*dx, *grads.values()])
    assert all(torch.equal(a, b) for a, b in zip(*seen))


def test_rows_of_zeros_and_what_is_not_finite():
    """A row of zeros stays zero under a norm; NaN and infinities stay in their row, and beside a channel that does not turn, in it."""
    import torch

    p = Problem(B=1, nh=2, grid=(2, 2, 2), kind="rms", dims=(8, 10, 4), dtype="float32")
    x = p.x[0]
    x[0, 0, 1] = 0
    x[0, 0, 2, 5] = float("nan")
    x[0, 1, 3, 63] = float("inf")
    x[0, 1, 4] *= 1e25  # squares beyond binary32
    x[0, 1, 5] *= 1e-25
    with np.errstate(invalid="ignore"):
        want = p.forward(0)
    out = p.empty(2)
    _pb().paro_qk_norm_rope(p.s, p.axes, p.table, p.norm, x, p.x[1], *out)
    got = host(out[0])
    assert bool((out[0][0, 0, 1] == 0).all())
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want[0, 0, 2]).all() and np.isfinite(want[0, 1, 4]).all()
    fine = np.isfinite(want).all(-1)
    check_values(out[0].cpu()[torch.from_numpy(fine)], want[fine], p.dtype, "finite rows")
    rest = np.zeros((1, 2, 8, 64))
    rest[0, 1, 0, 60] = np.inf
    x.copy_(torch.from_numpy(rest))
    _pb().paro_rope(p.s, p.axes, p.table, x, out[0])
    assert np.array_equal(host(out[0]), rest)


QUANT = [
    dict(), dict(block=32), dict(d=128, kind="layer", T=64, text_norm=True, grid=(1, 8, 8)), dict(d=128, block=32, kind="rms", halves=1, dims=(44, 42, 42)),
    dict(kind="layer", layout="fused", grid=(3, 7, 11), nh=6), dict(kind="none", layout="tokens", halves=1, T=5, grid=(1, 5, 7)),
    dict(B=1, nh=1, grid=(1, 1, 1)), dict(B=1, nh=2, grid=(1, 1, 65), block=64, dims=(8, 10, 4)), dict(kind="layer", dims=(0, 0, 0), T=3),
    dict(kind="none", dims=(0, 0, 0)), dict(dims=(8, 8, 8), T=70, text_norm=True), dict(d=128, dims=(0, 0, 64), halves=1), dict(B=1, nh=12, grid=(5, 9, 10), dims=(20, 22, 22), kind="layer"),
]


def _buffers(pb, s, bits_qk, bits_pv, fill):
    import torch

    k = pb.paro_nblocks(s)
    codes = [torch.full(pb.codes_shape(s, b, lay), fill, dtype=torch.bfloat16 if b == 16 else torch.int8, device="cuda:0")
             for b, lay in ((bits_qk, pb.PARO_ROWS), (bits_qk, pb.PARO_ROWS), (bits_pv, pb.PARO_VT))]
    return codes, [torch.full((s.B, s.nh, k), float(fill), device="cuda:0") for _ in range(3)]


@pytest.mark.parametrize("bits", [(8, 8), (8, 4), (4, 4), (4, 8), (16, 16)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("case", QUANT, ids=_id)
def test_quantize(case, dtype, bits):
    """The codes and scales of the two calls it replaces, and those of the oracle."""
    import torch

    pb = _pb()
    p = Problem(dtype=dtype, **case)
    ids = (np.arange(p.nh) * 5 % 6).astype(np.uint8)
    got, gs = _buffers(pb, p.s, *bits, 2)
    pb.paro_qk_norm_rope_quantize_qkv(p.s, *bits, ids, p.axes, p.table, p.norm, *p.x, got[0], gs[0], got[1], gs[1], got[2], gs[2])
    wide = Problem(**dict(case, dtype="float32", layout="heads"))
    wide.norm = p.norm
    for a, b in zip(wide.x, p.x):
        a.copy_(b.float())
    out = wide.empty(2)
    pb.paro_qk_norm_rope(p.s, p.axes, p.table, p.norm, wide.x[0], wide.x[1], *out)
    want, ws = _buffers(pb, p.s, *bits, 1)
    pb.paro_permute_quantize_qkv(p.s, *bits, ids, *out, wide.x[2], want[0], ws[0], want[1], ws[1], want[2], ws[2])
    for i in range(3):
        assert torch.equal(got[i], want[i]) and torch.equal(gs[i], ws[i]), i
    if bits[0] != 8:
        return
    y = p.forward(0).astype(np.float32)
    for h in range(p.nh):
        idx = po.perm_index(*p.grid, p.T, int(ids[h]))
        codes, scales = po.prepare_operand(y[0, h], idx, pb.paro_npad(p.s), p.s.block, 8)
        assert np.array_equal(gs[0][0, h].cpu().numpy(), scales) and np.array_equal(got[0][0, h].cpu().numpy(), codes), h


@pytest.mark.parametrize("weight,bias", [(None, None), (-1.5, None), (-1.5, 0.0), (1.5, -0.0)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_signs_of_zeros(kind, weight, bias):
    """Rows that are their mean, rows of zeros of either sign: bf16 codes are those of the two calls in every bit, and so are the forward
    call's zeros: a bias that is not there is a zero, as one that is."""
    import torch

    pb = _pb()
    p = Problem(kind=kind, ones=True, dtype="float32", T=5, dims=(8, 0, 16), grid=(2, 3, 11))
    for i, x in enumerate(p.x[:2]):
        x[..., 0::4, :], x[..., 1::4, :], x[..., 2::4, :] = 0.0, -0.0, 0.5 - i
    vectors = {}
    for name, value in (("weight", weight), ("bias", bias)):
        if value is not None and (name == "weight" or kind == "layer"):
            vectors.update({x + "_" + name: torch.full((p.d,), value, device="cuda:0") for x in "qk"})
    norm = pb.QkNorm(pb.PARO_NORM_RMS if kind == "rms" else pb.PARO_NORM_LAYER, 1e-6, **vectors)
    ids = np.array([0, 3, 5], np.uint8)
    got, gs = _buffers(pb, p.s, 16, 16, 2)
    pb.paro_qk_norm_rope_quantize_qkv(p.s, 16, 16, ids, p.axes, p.table, norm, *p.x, got[0], gs[0], got[1], gs[1], got[2], gs[2])
    out = p.empty(2)
    pb.paro_qk_norm_rope(p.s, p.axes, p.table, norm, p.x[0], p.x[1], *out)
    want, ws = _buffers(pb, p.s, 16, 16, 1)
    pb.paro_permute_quantize_qkv(p.s, 16, 16, ids, *out, p.x[2], want[0], ws[0], want[1], ws[1], want[2], ws[2])
    for i in range(3):
        off = int((got[i].view(torch.int16) != want[i].view(torch.int16)).sum())
        assert off == 0, (i, off)
    if kind == "layer" and bias is None:
        for y in out:
            still = y[..., p.n_img:, :]  # text does not turn: (x - m) r w + 0, never -0
            assert not torch.any((still == 0) & torch.signbit(still))


def _same_as_two_calls(p, ids, bits, x):
    """Codes and scales of x, which neither norm nor rotation changes, against those of paro_permute_quantize_qkv, in every bit."""
    import torch

    pb = _pb()
    got, gs = _buffers(pb, p.s, *bits, 2)
    pb.paro_qk_norm_rope_quantize_qkv(p.s, *bits, ids, p.axes, p.table, p.norm, *x, got[0], gs[0], got[1], gs[1], got[2], gs[2])
    want, ws = _buffers(pb, p.s, *bits, 1)
    pb.paro_permute_quantize_qkv(p.s, *bits, ids, *x, want[0], ws[0], want[1], ws[1], want[2], ws[2])
    for i in range(3):
        off = (got[i] != want[i]).flatten(3).any(-1), gs[i].view(torch.int32) != ws[i].view(torch.int32)
        assert not any(bool(o.any()) for o in off), (i, [o.nonzero()[:4].tolist() for o in off])


@pytest.mark.parametrize("bits", [(8, 8), (8, 4), (4, 4), (4, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_any_size(d, bits):
    """Blocks of every binary exponent: the smallest subnormals, scales whose significand is all ones, the largest numbers; values half a
    step from a code among the others."""
    import torch

    p = Problem(B=1, nh=6, d=d, kind="none", grid=(1, 1, 32 * 277), dims=(0, 0, 0), dtype="float32", block=32)
    r = p.rng
    for x in p.x:
        exponent = np.arange(277) - 149  # 2^-149 .. 2^127
        top = np.ldexp(1 + r.random((6, 277)), exponent).astype(np.float32)
        qmax = 7.0 if bits[0] == 4 else 127.0
        top[5] = (np.ldexp(2 - 2.0**-23, exponent - 8) * qmax).astype(np.float32)  # amax / qmax is all ones, or next to it
        v = (r.random((6, 277, 32, d)) * 2 - 1) * top[..., None, None]
        halves = np.rint(r.random((6, 277, 32, d)) * 2 * qmax - qmax - 0.5) + 0.5
        v = np.where(r.random(v.shape) < 0.3, halves * (top / np.float32(qmax)).astype(np.float64)[..., None, None], v)
        v = np.clip(v, -top[..., None, None].astype(np.float64), top[..., None, None].astype(np.float64)).astype(np.float32)
        v[:, :, 7, 3] = -top
        x.copy_(torch.from_numpy(v.reshape(1, 6, 277 * 32, d)))
        assert bool(torch.isfinite(x).all())
    _same_as_two_calls(p, np.zeros(6, np.uint8), bits, p.x)


@pytest.mark.parametrize("bits", [(8, 8), (4, 4)])
@pytest.mark.parametrize("block", [32, 64])
def test_codes_of_what_is_not_finite(block, bits):
    """NaN and infinities in a block, one or a whole wavefront of them, without a norm: the scale and codes of paro_permute_quantize_qkv."""
    p = Problem(B=1, nh=3, kind="none", grid=(3, 8, 16), T=5, dims=(0, 0, 0), dtype="float32", block=block)
    nan, inf = float("nan"), float("inf")
    for i, x in enumerate(p.x):
        x[0, 0, 17 + i, 5] = nan
        x[0, 0, 70:78] = nan
        x[0, 1, 3] = -nan
        x[0, 1, 100, 63], x[0, 1, 101, 0] = inf, nan
        x[0, 2, 130:200] = nan
        x[0, 2, 300, 1] = -inf
        x[0, 2, -1] = nan
    _same_as_two_calls(p, np.array([0, 2, 5], np.uint8), bits, p.x)


@pytest.mark.parametrize("case", [dict(d=64, kind="layer", layout="fused"), dict(d=128, kind="rms", halves=1, dims=(44, 42, 42)), dict(d=64, kind="none", block=32)], ids=_id)
def test_quantize_many_blocks(case):
    """Workgroups that go through several blocks, from image tokens into text: the codes and scales of the two calls."""
    import torch

    pb = _pb()
    for bits in ((8, 8), (16, 16)):
        p = Problem(B=2, nh=48, grid=(2, 9, 125), T=200, text_norm=case["kind"] != "none", dtype="float32", **case)
        assert 3 * 2 * 48 * ((pb.paro_nblocks(p.s) + 1) // 2) >= 4096  # two blocks or more each
        ids = (np.arange(48) % 6).astype(np.uint8)
        got, gs = _buffers(pb, p.s, *bits, 2)
        pb.paro_qk_norm_rope_quantize_qkv(p.s, *bits, ids, p.axes, p.table, p.norm, *p.x, got[0], gs[0], got[1], gs[1], got[2], gs[2])
        y = [torch.empty((2, 48, p.n, p.d), device="cuda:0") for _ in range(2)]
        pb.paro_qk_norm_rope(p.s, p.axes, p.table, p.norm, p.x[0], p.x[1], *y)
        want, ws = _buffers(pb, p.s, *bits, 1)
        pb.paro_permute_quantize_qkv(p.s, *bits, ids, *y, p.x[2].contiguous(), want[0], ws[0], want[1], ws[1], want[2], ws[2])
        for i in range(3):
            assert torch.equal(got[i], want[i]) and torch.equal(gs[i], ws[i]), i


def test_a_layer_from_projections_to_attention():
    """ParoAttention on Q, K, V as a projection leaves them: the bits of norms and rotation, then the fused layer."""
    import torch

    from paper_2506_16054_amd import workloads as wl
    from paper_2506_16054_amd.pipeline import ParoAttention, QkNormRope

    pb = _pb()
    for block, d, dtype in ((64, 64, "float32"), (32, 128, "float32"), (64, 128, "bfloat16")):
        p = Problem(B=2, nh=4, d=d, grid=(2, 8, 8), T=64, kind="rms", text_norm=True, layout="fused", dtype=dtype, block=block)
        k = pb.paro_nblocks(p.s)
        live = np.random.default_rng(4).random((4, k, k)) < 0.7
        live[:, np.arange(k), np.arange(k)] = True
        pa = ParoAttention(p.s, np.array([0, 2, 3, 5], np.uint8), wl.pack_bitmask(live), 8, 8, p.dtype)
        step = QkNormRope(p.s, p.dims, norm=p.norm)
        assert torch.equal(step.table, p.table)
        o = pa.run_norm_rope(step, *p.x).clone()
        y = [torch.empty((2, 4, p.n, d), device="cuda:0") for _ in range(2)]
        pb.paro_qk_norm_rope(p.s, step.axes, step.table, p.norm, p.x[0].float(), p.x[1].float(), *y)
        assert torch.equal(pa.run_fused(*y, p.x[2].float().contiguous()), o)
        q, kk = step.forward(p.x[0], p.x[1])  # what a program does that looks at Q and K
        check_values(q, p.forward(0), p.dtype, "forward")
        dq, dk = step.backward(p.x[0], p.x[1], q, kk, pb.QkNormGrad(q_weight=torch.empty((d,), device="cuda:0")))
        assert dq.shape == q.shape and bool(torch.isfinite(dk.float()).all())


@pytest.mark.parametrize("what", ["forward", "backward", "quantize"])
def test_streams_and_graphs(what):
    """On a side stream behind inputs that arrive late, and captured: every replay gives what the eager call gives, with eager work
    between the replays."""
    import torch

    pb = _pb()
    p = Problem(B=1, nh=4, grid=(3, 7, 11), kind="layer", T=9, text_norm=True, dtype="float32")
    dy = p.rows(2)
    grads = {name: torch.empty((p.d,), device="cuda:0") for name in p.vectors}
    scratch = torch.empty((pb.paro_qk_norm_rope_backward_bytes(p.s),), dtype=torch.uint8, device="cuda:0")
    codes, scales = _buffers(pb, p.s, 8, 8, 0)
    out = p.empty(2)
    x = [torch.zeros_like(t) for t in p.x]

    def call():
        if what == "forward":
            pb.paro_qk_norm_rope(p.s, p.axes, p.table, p.norm, x[0], x[1], *out)
            return out
        if what == "backward":
            pb.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm, x[0], x[1], *dy, *out, pb.QkNormGrad(**grads), scratch)
            return [*out, *grads.values()]
        pb.paro_qk_norm_rope_quantize_qkv(p.s, 8, 8, [0, 1, 4, 5], p.axes, p.table, p.norm, *x, codes[0], scales[0], codes[1], scales[1], codes[2], scales[2])
        return [*codes, *scales]

    def fresh(seed):
        return [t + 0.01 * seed for t in p.x]

    def load(values):
        for a, b in zip(x, values):
            a.copy_(b)

    load(fresh(0))
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for t in x:
            t.zero_()
        torch.cuda._sleep(20_000_000)  # some 10 ms
        load(fresh(0))
        got = [t.clone() for t in call()]
        side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (1, 2, 3):
        load(fresh(seed))
        want = [t.clone() for t in call()]
        for t in (*out, *codes, *scales, *grads.values(), scratch):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        after = [*out] if what == "forward" else [*out, *grads.values()] if what == "backward" else [*codes, *scales]
        assert all(torch.equal(a, b) for a, b in zip(after, want)), seed


def test_the_native_module_takes_the_calls():
    """What it is made for it does not leave to the binding."""
    import torch

    pb = _pb()
    f = pb._native()
    for layout in ("heads", "fused"):
        p = Problem(kind="layer", T=3, text_norm=True, layout=layout)
        out, dy = p.empty(2), p.rows(2)
        grads = pb.QkNormGrad(**{name: torch.empty((64,), device="cuda:0") for name in p.vectors})
        scratch = torch.empty((pb.paro_qk_norm_rope_backward_bytes(p.s),), dtype=torch.uint8, device="cuda:0")
        codes, scales = _buffers(pb, p.s, 8, 4, 0)
        ids = np.array([0, 1, 2], np.uint8)
        assert f.paro_rope(p.s, p.axes, p.table, p.x[0], out[0], True) == pb.PARO_OK
        assert f.paro_qk_norm_rope(p.s, p.axes, p.table, p.norm._native, *p.x[:2], *out) == pb.PARO_OK
        assert f.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm._native, *p.x[:2], *dy, *out, grads._vectors, scratch) == pb.PARO_OK
        assert f.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm._native, *p.x[:2], *dy, *out, None, None) == pb.PARO_OK
        assert f.paro_qk_norm_rope_quantize_qkv(p.s, 8, 4, ids, p.axes, p.table, p.norm._native, *p.x, codes[0], scales[0], codes[1], scales[1], codes[2],
                                                scales[2]) == pb.PARO_OK
        # and declines what the binding refuses
        for bad in (p.x[0].cpu(), p.x[0].half(), p.x[0][..., ::2], p.x[0][:, :, 1:], None):
            assert f.paro_rope(p.s, p.axes, p.table, bad, out[0], False) is None
            assert f.paro_qk_norm_rope(p.s, p.axes, p.table, p.norm._native, p.x[0], bad, *out) is None
        assert f.paro_rope(p.s, p.axes, p.table[1:], p.x[0], out[0], False) is None and f.paro_rope(p.s, p.s, p.table, p.x[0], out[0], False) is None
        assert f.paro_qk_norm_rope(p.s, p.axes, p.table, p.norm._native[:-1], *p.x[:2], *out) is None
        assert f.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm._native, *p.x[:2], *dy, *out, grads._vectors, scratch[:-4]) is None


def test_refusals_of_the_binding():
    import torch

    pb = _pb()
    p = Problem()
    out = p.empty(2)
    f = lambda q, *rest, norm=p.norm, table=p.table: pb.paro_qk_norm_rope(p.s, p.axes, table, norm, q, *(rest or (p.x[1], *out)))
    wide = torch.zeros((2, 3, p.n, 128), dtype=p.dtype, device="cuda:0")
    for bad in (p.x[0].cpu(), p.x[0].float(), p.x[0].half(), p.x[0][:, :, 1:], wide[..., ::2], wide.view(-1)[4: 4 + p.x[0].numel()].view(p.x[0].shape)):
        with pytest.raises(pb.ParoError):
            f(bad)
    with pytest.raises(pb.ParoError):
        f(p.x[0], p.x[1], out[0], p.x[1][:, :1].expand(-1, 3, -1, -1))  # one row for three heads
    with pytest.raises(pb.ParoError):
        f(p.x[0], p.x[1], out[0], out[0])
    with pytest.raises(pb.ParoError):
        f(p.x[0], table=p.table[:-1])
    with pytest.raises(pb.ParoError):
        f(p.x[0], table=None)
    for vector in (torch.zeros((32,), device="cuda:0"), torch.zeros((64,)), torch.zeros((64,), dtype=torch.bfloat16, device="cuda:0"),
                   torch.zeros((65,), device="cuda:0")[1:]):
        with pytest.raises(pb.ParoError):
            f(p.x[0], norm=pb.QkNorm(pb.PARO_NORM_RMS, 1e-6, q_weight=vector))
    f(p.x[0][:, :1].expand(-1, 3, -1, -1))  # an input that heads share is read as it stands
    grad = pb.QkNormGrad(q_weight=torch.zeros((64,), device="cuda:0"))
    for scratch in (None, torch.empty((16,), dtype=torch.uint8, device="cuda:0")):
        with pytest.raises(pb.ParoError):
            pb.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm, p.x[0], p.x[1], *out, *p.empty(2), grad, scratch)
    codes, scales = _buffers(pb, p.s, 8, 8, 0)
    with pytest.raises(pb.ParoError):
        pb.paro_qk_norm_rope_quantize_qkv(p.s, 8, 4, [0, 1, 2], p.axes, p.table, p.norm, *p.x, codes[0], scales[0], codes[1], scales[1], codes[2], scales[2])
    with pytest.raises(pb.ParoError):
        pb.paro_qk_norm_rope_quantize_qkv(p.s, 8, 8, [0, 1, 9], p.axes, p.table, p.norm, *p.x, codes[0], scales[0], codes[1], scales[1], codes[2], scales[2])


def _between(shape, dtype, mark):
    """A tensor with 64 marked elements in front of it and behind it, and a check that they are still there."""
    import torch

    n = int(np.prod(shape))
    whole = torch.full((n + 128,), mark, dtype=dtype, device="cuda:0")
    return whole[64: 64 + n].view(shape), lambda: bool((whole[:64] == mark).all()) and bool((whole[64 + n:] == mark).all())


@pytest.mark.parametrize("case", [dict(d=64, kind="layer", grid=(1, 5, 13), T=3), dict(d=128, kind="rms", grid=(1, 1, 1)), dict(d=64, kind="rms", block=32, grid=(3, 7, 5))],
                         ids=_id)
def test_nothing_beside_the_outputs_is_written(case):
    import torch

    pb = _pb()
    p = Problem(B=1, nh=3, dtype="float32", **case)
    intact, make = [], lambda shape, dtype, mark: (lambda t, ok: (intact.append(ok), t)[1])(*_between(shape, dtype, mark))
    shape = (1, 3, p.n, p.d)
    out = [make(shape, torch.float32, 7.0) for _ in range(2)]
    pb.paro_rope(p.s, p.axes, p.table, p.x[0], out[0])
    pb.paro_qk_norm_rope(p.s, p.axes, p.table, p.norm, *p.x[:2], *out)
    grads = {name: make((p.d,), torch.float32, 7.0) for name in p.vectors}
    scratch = make((pb.paro_qk_norm_rope_backward_bytes(p.s),), torch.uint8, 7)
    pb.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm, *p.x[:2], *p.rows(2), *out, pb.QkNormGrad(**grads), scratch)
    for bits in ((8, 8), (4, 4), (16, 16)):
        ct = torch.bfloat16 if bits[0] == 16 else torch.int8
        codes = [make(pb.codes_shape(p.s, bits[0], lay), ct, 7) for lay in (pb.PARO_ROWS, pb.PARO_ROWS, pb.PARO_VT)]
        scales = [make((1, 3, pb.paro_nblocks(p.s)), torch.float32, 7.0) for _ in range(3)]
        pb.paro_qk_norm_rope_quantize_qkv(p.s, *bits, [0, 3, 5], p.axes, p.table, p.norm, *p.x, codes[0], scales[0], codes[1], scales[1], codes[2], scales[2])
    assert all(ok() for ok in intact)


def test_two_streams_at_once():
    """Two gradients at the same time, each with a scratch of its own, give what each gives alone."""
    import torch

    pb = _pb()
    problems = [Problem(B=1, nh=8, grid=(4, 16, 17), kind="layer", dtype="float32", seed=s) for s in (1, 2)]
    work = []
    for p in problems:
        grads = {name: torch.empty((p.d,), device="cuda:0") for name in p.vectors}
        scratch = torch.empty((pb.paro_qk_norm_rope_backward_bytes(p.s),), dtype=torch.uint8, device="cuda:0")
        work.append((p, p.rows(2), p.empty(2), grads, scratch))

    def call(p, dy, dx, grads, scratch):
        pb.paro_qk_norm_rope_backward(p.s, p.axes, p.table, p.norm, *p.x[:2], *dy, *dx, pb.QkNormGrad(**grads), scratch)

    want = []
    for w in work:
        call(*w)
        want.append([t.clone() for t in (*w[2], *w[3].values())])
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, w in zip(streams, work):
            with torch.cuda.stream(stream):
                call(*w)
    torch.cuda.synchronize()
    for w, ref in zip(work, want):
        assert all(torch.equal(a, b) for a, b in zip((*w[2], *w[3].values()), ref))


@pytest.mark.parametrize("grid,T", [((1, 1, 1 << 20), 13), ((1 << 20, 1, 1), 0), ((3, 1021, 349), 70)])
def test_long_sequences(grid, T):
    """A million tokens: sampled rows against the oracle, the codes of one head against the two calls."""
    import torch

    pb = _pb()
    d, dims, n = 64, (16, 24, 24), int(np.prod(grid)) + T
    s, axes = pb.make_shape(1, 1, d, *grid, T, 64), pb.make_rope_axes((16, 24, 24))
    pos = [np.arange(x, dtype=np.float64) for x in grid]
    freq = [10000.0 ** (-np.arange(0, x, 2, dtype=np.float64) / x) for x in dims]
    h_table = pb.paro_rope_table(s, axes, pos, freq)
    table, norm = torch.from_numpy(h_table).to("cuda:0"), pb.QkNorm(pb.PARO_NORM_RMS, 1e-6)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    q, k, v = (torch.randn((1, 1, n, d), generator=gen, device="cuda:0") for _ in range(3))
    out = [torch.empty_like(q) for _ in range(2)]
    pb.paro_qk_norm_rope(s, axes, table, norm, q, k, *out)
    rng = np.random.default_rng(5)
    rows = np.unique(np.concatenate([[0, 1, n // 2, n - T - 1, n - 1], rng.integers(0, n, 200)]))
    cos, sin = np.ones((len(rows), d // 2)), np.zeros((len(rows), d // 2))
    for i, row in enumerate(rows):
        if row < n - T:
            coords, p, base = (row // (grid[1] * grid[2]), row // grid[2] % grid[1], row % grid[2]), 0, 0
            for c, extent, dim in zip(coords, grid, dims):
                part = h_table[base + c * (dim // 2): base + (c + 1) * (dim // 2)]
                cos[i, p: p + dim // 2], sin[i, p: p + dim // 2] = part[:, 0], part[:, 1]
                p, base = p + dim // 2, base + extent * (dim // 2)
    at = torch.from_numpy(rows).to("cuda:0")
    for x, y in zip((q, k), out):
        check_values(y[0, 0, at], on.norm_rope(host(x[0, 0, at]), "rms", 1e-6, 1.0, 0.0, cos, sin, 0), torch.float32, "rows")
    for order in (1, 5):
        got, gs = _buffers(pb, s, 8, 8, 2)
        want, ws = _buffers(pb, s, 8, 8, 1)
        pb.paro_qk_norm_rope_quantize_qkv(s, 8, 8, [order], axes, table, norm, q, k, v, got[0], gs[0], got[1], gs[1], got[2], gs[2])
        pb.paro_permute_quantize_qkv(s, 8, 8, [order], *out, v, want[0], ws[0], want[1], ws[1], want[2], ws[2])
        for i in range(3):
            assert torch.equal(got[i], want[i]) and torch.equal(gs[i], ws[i]), (order, i)


def test_offsets_beyond_32_bits():
    """A batch stride of more than 2^32 bytes."""
    import torch

    p = Problem(B=1, nh=2, grid=(2, 3, 5), kind="rms")
    far = torch.empty((2, (1 << 31) + (1 << 20)), dtype=torch.bfloat16, device="cuda:0")
    rows = [far[:, at: at + 2 * 30 * 64].view(2, 2, 30, 64) for at in ((1 << 31), (1 << 31) + (1 << 16))]
    pb = _pb()
    s = pb.make_shape(2, 2, 64, 2, 3, 5, 0, 64)
    for t, x in zip(rows, p.x):
        t.copy_(x.expand(2, -1, -1, -1))
    rows[0][1] *= 2
    pb.paro_qk_norm_rope(s, p.axes, p.table, p.norm, *rows, *rows)
    p.x[0] *= 2
    check_values(rows[0][1], p.forward(0)[0], p.dtype, "second batch")
    check_values(rows[1][1], p.forward(1)[0], p.dtype, "second batch")
