"""What is timed of the operators in front of the attention call: the norms of Q and K per head, the rotation by the token's
(frame, height, width) position, their backward pass, and both together with the reorder and the block quantizer.

A case is a dict of plain values.  ``op`` says which call:

  rope       one tensor rotated; ``inverse`` is the direction of the backward pass
  norm_rope  Q and K normalised per head and rotated
  backward   the gradients of norm_rope: of Q, of K and of the norms' weights (and biases)
  quantize   norm_rope of Q and K, and Q, K, V reordered and quantized for the attention kernels

``layout`` is how Q, K, V lie in memory: "heads" [B, nh, N, d], or "fused", views of the output [B, N, 3, nh, d] of one
projection.  ``norm`` is "none", "rms" or "layer"; with ``text_norm`` the text tokens have weights of their own (joint layers,
where text comes from its own projection).  ``d0, d1, d2`` channels turn with the frame, height and width position, ``pairs``
says which channels form a pair.  Positions are ``start + step * index``.

Where ``own`` is false the operators are elementary torch operations in 32 bits (in 64 for the values that are rounded to codes and
for the long sums of the weights' gradients); where it is true they are the package's calls."""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
THETA = 10000.0


# ---- cases ---------------------------------------------------------------------------------------------------------
def _case(op, B, nh, d, grid, T_text, dims, dtype, norm="none", pairs="adjacent", layout="heads", text_norm=False, inverse=False, bits=16, block=64,
          start=0.0, step=1.0):
    F, Hg, Wg = grid
    return {"op": op, "B": B, "nh": nh, "d": d, "F": F, "Hg": Hg, "Wg": Wg, "T_text": T_text, "d0": dims[0], "d1": dims[1], "d2": dims[2],
            "pairs": pairs, "dtype": dtype, "norm": norm, "layout": layout, "text_norm": text_norm, "inverse": inverse, "bits": bits, "block": block,
            "start": start, "step": step}


def listed():
    video = (13, 30, 45)  # 17550 latent tokens
    image = (1, 64, 64)   # 4096 image tokens + 512 text tokens
    v64, v128 = (16, 24, 24), (16, 56, 56)
    cases = {
        # the smallest layer the tests and smoke() run: launches and host work are all of it
        "rope_tiny_f32": _case("rope", 1, 2, 64, (2, 8, 8), 0, v64, "f32"),
        # the headline layer's Q, read where the projection of Q, K, V left it
        "rope_video48": _case("rope", 1, 48, 64, video, 0, v64, "bf16", layout="fused"),
        # the backward direction on an image model's joint layer; uneven axes and pairs across the halves of a head, positions far out
        "rope_image24_inverse": _case("rope", 1, 24, 128, image, 512, (44, 42, 42), "bf16", pairs="halves", inverse=True, start=20000.0),
        # one token of one frame, as a stream of single latents is extended
        "norm_rope_one_token": _case("norm_rope", 1, 24, 128, (1, 1, 1), 0, v128, "bf16", norm="rms", layout="fused", start=977.0),
        # a video layer: layer norm with bias, Q and K from the fused projection
        "norm_rope_video48": _case("norm_rope", 1, 48, 64, video, 0, v64, "bf16", norm="layer", layout="fused"),
        # a joint layer: root-mean-square norms, text tokens with weights of their own
        "norm_rope_image24": _case("norm_rope", 1, 24, 128, image, 512, v128, "bf16", norm="rms", text_norm=True),
        # a small batch of ragged layers in fp32
        "norm_rope_ragged_f32": _case("norm_rope", 2, 6, 64, (5, 17, 23), 0, (20, 22, 22), "f32", norm="rms", pairs="halves", step=0.5),
        # training steps of the same layers
        "backward_video48": _case("backward", 1, 48, 64, video, 0, v64, "bf16", norm="layer", layout="fused"),
        "backward_image24": _case("backward", 1, 24, 128, image, 512, v128, "bf16", norm="rms", text_norm=True),
        "backward_ragged_f32": _case("backward", 2, 6, 64, (5, 17, 23), 0, (20, 22, 22), "f32", norm="layer", pairs="halves"),
        # what a layer runs in front of the 8-bit attention kernel, and of the unquantized one
        "quantize_image24_int8": _case("quantize", 1, 24, 128, image, 512, v128, "bf16", norm="rms", text_norm=True, bits=8),
        "quantize_video48_bf16": _case("quantize", 1, 48, 64, video, 0, v64, "bf16", norm="layer", layout="fused"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _tokens(c):
    return c["F"] * c["Hg"] * c["Wg"] + c["T_text"]


def _elements(c):
    return c["B"] * c["nh"] * _tokens(c) * c["d"]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    most = max(_elements(c) for c in listed())
    while True:
        op = rng.choice(["rope", "norm_rope", "norm_rope", "backward", "backward", "quantize"])
        d = rng.choice([64, 64, 128])
        dims = rng.choice([(16, 24, 24), (20, 22, 22), (0, 32, 32), (8, 16, 16)] if d == 64 else [(16, 56, 56), (32, 48, 48), (44, 42, 42), (0, 64, 64)])
        block = rng.choice([64, 64, 32])
        grid = (rng.choice([1, 1, 2, 5, 9, 13, 16]), _log_int(rng, 1, 64), _log_int(rng, 1, 64))
        text = rng.choice([0, 0, 226, 512])
        if op == "quantize" and (grid[0] * grid[1] * grid[2]) % block:
            text = 0  # text tokens follow whole image blocks
        norm = rng.choice(["rms", "rms", "layer", "none"]) if op in ("norm_rope", "quantize") else rng.choice(["rms", "layer"])
        c = _case(op, rng.choice([1, 1, 2, 3]), _log_int(rng, 1, 48), d, grid, text, dims, rng.choice(["bf16", "bf16", "f32"]),
                  "none" if op == "rope" else norm, rng.choice(["adjacent", "halves"]), rng.choice(["heads", "fused"]),
                  bool(text) and norm != "none" and op != "rope" and rng.random() < 0.5, op == "rope" and rng.random() < 0.5,
                  rng.choice([8, 16]), block, float(rng.choice([0, 0, 30, 5000])), rng.choice([1.0, 1.0, 0.5, 0.75]))
        if _elements(c) * (2 if c["dtype"] == "f32" else 1) <= most:
            return c


# ---- inputs --------------------------------------------------------------------------------------------------------
def _table(c):
    """Cosine and sine, float32, of position x frequency in 64 bits: entry (i, p) of an axis is its i-th coordinate and p-th pair; the
    axes' entries one behind the other."""
    parts = []
    for dim, extent in zip((c["d0"], c["d1"], c["d2"]), (c["F"], c["Hg"], c["Wg"])):
        if dim:
            freq = THETA ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=DEV) / dim)
            pos = c["start"] + c["step"] * torch.arange(extent, dtype=torch.float64, device=DEV)
            angle = pos[:, None] * freq
            parts.append(torch.stack([angle.cos(), angle.sin()], -1).float())  # [extent, dim / 2, 2]
    return parts


def _per_token(c, parts):
    """The table spread over the tokens: cosine and sine [N, d / 2]; pairs that no axis turns and text tokens have (1, 0)."""
    F, Hg, Wg, n = c["F"], c["Hg"], c["Wg"], _tokens(c)
    cs = torch.zeros((n, c["d"] // 2, 2), device=DEV)
    cs[..., 0] = 1.0
    grid, p0, views = cs[: F * Hg * Wg].view(F, Hg, Wg, c["d"] // 2, 2), 0, ((F, 1, 1), (1, Hg, 1), (1, 1, Wg))
    parts = list(parts)
    for dim, view in zip((c["d0"], c["d1"], c["d2"]), views):
        if dim:
            part = parts.pop(0)
            grid[..., p0: p0 + dim // 2, :] = part.view(*view, dim // 2, 2)
            p0 += dim // 2
    return cs[..., 0].contiguous(), cs[..., 1].contiguous()


def _reordered(c, perm_id):
    """Default-order positions of a head's tokens in the order `perm_id` of the grid's axes; text tokens stay behind."""
    F, Hg, Wg, n = c["F"], c["Hg"], c["Wg"], _tokens(c)
    order = ((0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0))[perm_id]
    at = torch.arange(F * Hg * Wg, device=DEV).view(F, Hg, Wg).permute(*order).reshape(-1)
    return torch.cat([at, torch.arange(F * Hg * Wg, n, device=DEV)])


def _slots(block):
    """Where token i of a block of V stands in the order that the attention kernel's products take keys in."""
    i = torch.arange(block, device=DEV)
    return (i & ~31) | ((i & 4) << 2) | ((i & 24) >> 1) | (i & 3)


def prepare(case, seed):
    c = {k: v for k, v in case.items() if k != "name"}
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    B, nh, d, n, block = c["B"], c["nh"], c["d"], _tokens(c), c["block"]
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    k = -(-n // block)
    z = dict(device=DEV)
    # what a projection gives: channels of different size with an offset, tokens of different norm
    size = torch.exp(0.5 * torch.randn((3, nh, d), generator=gen, **z))
    offset = 0.5 * torch.randn((3, nh, d), generator=gen, **z)
    count = 1 if c["op"] == "rope" else 3 if c["op"] == "quantize" else 2

    def activations():
        if c["layout"] == "fused":
            whole = torch.randn((B, n, 3, nh, d), generator=gen, **z)
            whole.mul_(torch.exp(0.3 * torch.randn((B, n, 1, 1, 1), generator=gen, **z))).mul_(size).add_(offset)
            return list(whole.to(dtype).permute(2, 0, 3, 1, 4)[:count])
        return [(torch.randn((B, nh, n, d), generator=gen, **z) * torch.exp(0.3 * torch.randn((B, 1, n, 1), generator=gen, **z)) * size[i][:, None]
                 + offset[i][:, None]).to(dtype) for i in range(count)]

    x = activations()
    parts = _table(c)
    state = {"case": c, "x": x, "table": torch.cat([p.reshape(-1, 2) for p in parts]) if parts else None}
    state["cos"], state["sin"] = _per_token(c, parts)
    state["out"] = [torch.empty((B, nh, n, d), dtype=dtype, **z) for _ in range(0 if c["op"] == "quantize" else min(count, 2))]
    names = []
    if c["norm"] != "none":
        kinds = ["weight"] + (["bias"] if c["norm"] == "layer" else [])
        names = ["%s%s_%s" % (t, x, kind) for t in (("", "text_") if c["text_norm"] else ("",)) for x in "qk" for kind in kinds]
    state["norm"] = {name: (1.0 if name.endswith("weight") else 0.0) + 0.3 * torch.randn((d,), generator=gen, **z) for name in names}
    if c["op"] == "backward":
        state["dy"] = [torch.randn((B, nh, n, d), generator=gen, **z).to(dtype) for _ in range(2)]
        if c["layout"] == "fused":
            state["dx"] = list(torch.empty((B, n, 3, nh, d), dtype=dtype, **z).permute(2, 0, 3, 1, 4)[:2])
        else:
            state["dx"] = [torch.empty((B, nh, n, d), dtype=dtype, **z) for _ in range(2)]
        state["dnorm"] = {name: torch.empty((d,), **z) for name in names}
    if c["op"] == "quantize":
        state["perm_ids"] = np.random.default_rng(int(seed)).integers(0, 6, size=nh).astype(np.uint8)
        state["at"] = torch.stack([_reordered(c, int(p)) for p in state["perm_ids"]])  # [nh, N]
        ct = torch.bfloat16 if c["bits"] == 16 else torch.int8
        rows, vt = (B, nh, k * block, d), (B, nh, k, d, block)
        state["codes"] = [torch.empty(shape, dtype=ct, **z) for shape in (rows, rows, vt)]
        state["scales"] = [torch.empty((B, nh, k), **z) for _ in range(3)]
    return state


# ---- one pass, plain -----------------------------------------------------------------------------------------------
def _pair(c, u):
    """The two channels of every pair: [..., d / 2] each."""
    return (u[..., 0::2], u[..., 1::2]) if c["pairs"] == "adjacent" else (u[..., : c["d"] // 2], u[..., c["d"] // 2:])


def _unpair(c, a, b):
    return torch.stack([a, b], -1).flatten(-2) if c["pairs"] == "adjacent" else torch.cat([a, b], -1)


def _rotated(state, u, inverse=False):
    c, cos, sin = state["case"], state["cos"].to(u.dtype), state["sin"].to(u.dtype)
    if inverse:
        sin = -sin
    a, b = _pair(c, u)
    return _unpair(c, a * cos - b * sin, a * sin + b * cos)


def _per_row(state, name, dtype):
    """A norm's weight or bias for every token: [1, d], or [N, d] where text tokens have their own."""
    c, w = state["case"], state["norm"][name].to(dtype)
    if not c["text_norm"]:
        return w[None]
    n_img = _tokens(c) - c["T_text"]
    return torch.cat([w[None].expand(n_img, -1), state["norm"]["text_" + name].to(dtype)[None].expand(c["T_text"], -1)])


def _normed(state, which, x):
    """(value divided by its norm, 1 / norm) of every row, and the row behind the weights."""
    c = state["case"]
    if c["norm"] == "none":
        return None, None, x
    if c["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    xhat = x * r
    u = xhat * _per_row(state, which + "_weight", x.dtype)
    if c["norm"] == "layer":
        u = u + _per_row(state, which + "_bias", x.dtype)
    return xhat, r, u


def _backward(state, which, x, dy, dtype):
    c, grads = state["case"], {}
    xhat, r, _ = _normed(state, which, x.float())
    g = _rotated(state, dy.float(), inverse=True)
    n_img = _tokens(c) - c["T_text"]
    spans = {"": slice(0, n_img), "text_": slice(n_img, None)} if c["text_norm"] else {"": slice(None)}
    for prefix, span in spans.items():
        grads[prefix + which + "_weight"] = (g[:, :, span] * xhat[:, :, span]).double().sum((0, 1, 2)).float()
        if c["norm"] == "layer":
            grads[prefix + which + "_bias"] = g[:, :, span].double().sum((0, 1, 2)).float()
    du = g * _per_row(state, which + "_weight", torch.float32)
    dx = du - xhat * (du * xhat).mean(-1, keepdim=True)
    if c["norm"] == "layer":
        dx = dx - du.mean(-1, keepdim=True)
    return (r * dx).to(dtype), grads


def _quantized(state, y, transposed):
    """The values that the codes of reordered blocks stand for, in the layout of the codes, and the scales.  y: [B, nh, N, d] as
    float32; blocks of `block` tokens share a scale."""
    c = state["case"]
    B, nh, n, d, block = c["B"], c["nh"], _tokens(c), c["d"], c["block"]
    k = -(-n // block)
    y = torch.take_along_dim(y, state["at"][None, :, :, None], 2)
    padded = torch.zeros((B, nh, k * block, d), device=DEV)
    padded[:, :, :n] = y
    y = padded.view(B, nh, k, block, d)
    if c["bits"] == 16:
        values, scale = y.to(torch.bfloat16), None
    else:
        amax = y.abs().amax((-1, -2))
        scale = torch.where(amax > 0, (amax.double() / 127.0).float(), torch.ones_like(amax))
        quotient = (y.double() / scale[..., None, None].double()).float()  # one rounding to 32 bits, as of a 32-bit divide
        values = torch.round(quotient).clamp(-127, 127) * scale[..., None, None]
    if transposed:
        values, by_token = torch.empty_like(values.transpose(-1, -2), memory_format=torch.contiguous_format), values.transpose(-1, -2)
        values[..., _slots(block)] = by_token
    else:
        values = values.view(B, nh, k * block, d)
    return values if scale is None else (values, scale)


def _plain(state):
    c, x = state["case"], state["x"]
    dtype = x[0].dtype
    if c["op"] == "rope":
        return _rotated(state, x[0].float(), c["inverse"]).to(dtype)
    if c["op"] == "norm_rope":
        return [_rotated(state, _normed(state, which, x[i].float())[2]).to(dtype) for i, which in enumerate("qk")]
    if c["op"] == "backward":
        dq, grads = _backward(state, "q", x[0], state["dy"][0], dtype)
        dk, more = _backward(state, "k", x[1], state["dy"][1], dtype)
        return {"dq": dq, "dk": dk, **grads, **more}
    # codes are decisions at borders: what is rounded to them is computed in 64 bits and rounded to 32 once
    y = [_rotated(state, _normed(state, which, x[i].double())[2]).float() for i, which in enumerate("qk")]
    return [_quantized(state, y[0], False), _quantized(state, y[1], False), _quantized(state, x[2].float(), True)]


# ---- one pass, the package's calls ---------------------------------------------------------------------------------
def _plan(state):
    """What a program keeps per layer: the shape, the axes and the norms."""
    from paper_2506_16054_amd import binding as pb

    c = state["case"]
    plan = {"s": pb.make_shape(c["B"], c["nh"], c["d"], c["F"], c["Hg"], c["Wg"], c["T_text"], c["block"]),
            "axes": pb.make_rope_axes((c["d0"], c["d1"], c["d2"]), pb.PARO_PAIRS_ADJACENT if c["pairs"] == "adjacent" else pb.PARO_PAIRS_HALVES),
            "norm": pb.QkNorm({"none": pb.PARO_NORM_NONE, "rms": pb.PARO_NORM_RMS, "layer": pb.PARO_NORM_LAYER}[c["norm"]], EPS, **state["norm"])}
    if c["op"] == "backward":
        plan["grads"] = pb.QkNormGrad(**state["dnorm"])
        plan["scratch"] = torch.empty((pb.paro_qk_norm_rope_backward_bytes(plan["s"]),), dtype=torch.uint8, device=DEV)
    return plan


def _own(state):
    from paper_2506_16054_amd import binding as pb

    c, x = state["case"], state["x"]
    if "plan" not in state:
        state["plan"] = _plan(state)
    plan = state["plan"]
    s, axes, norm, table = plan["s"], plan["axes"], plan["norm"], state["table"]
    if c["op"] == "rope":
        pb.paro_rope(s, axes, table, x[0], state["out"][0], c["inverse"])
        return state["out"][0]
    if c["op"] == "norm_rope":
        pb.paro_qk_norm_rope(s, axes, table, norm, x[0], x[1], *state["out"])
        return state["out"]
    if c["op"] == "backward":
        pb.paro_qk_norm_rope_backward(s, axes, table, norm, x[0], x[1], *state["dy"], *state["dx"], plan["grads"], plan["scratch"])
        return {"dq": state["dx"][0], "dk": state["dx"][1], **state["dnorm"]}
    bits, (qc, kc, vc), (sq, sk, sv) = c["bits"], state["codes"], state["scales"]
    pb.paro_qk_norm_rope_quantize_qkv(s, bits, bits, state["perm_ids"], axes, table, norm, *x, qc, sq, kc, sk, vc, sv)
    if bits == 16:
        return [qc, kc, vc]
    # what the codes stand for: a program would hand them to the attention call as they are
    return [(torch.mul(codes.view(*scale.shape, -1), scale[..., None]).view(codes.shape), scale) for codes, scale in ((qc, sq), (kc, sk), (vc, sv))]


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition, in 64 bits ------------------------------------------------------------------------------------
def _turned(state, u, sign=1.0):
    """Pairs as complex numbers, each times the unit number of its token and frequency."""
    c = state["case"]
    unit = torch.complex(state["cos"].double(), sign * state["sin"].double())
    if c["pairs"] == "adjacent":
        z = torch.view_as_complex(u.reshape(*u.shape[:-1], c["d"] // 2, 2).contiguous()) * unit
        return torch.view_as_real(z).reshape(u.shape)
    lo, hi = u.split(c["d"] // 2, -1)
    z = torch.complex(lo.contiguous(), hi.contiguous()) * unit
    return torch.cat([z.real, z.imag], -1)


def _forward64(state, which, x, norm):
    c = state["case"]
    if c["norm"] != "none":
        n_img = _tokens(c) - c["T_text"]
        if c["norm"] == "rms":
            x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["d"] + EPS)
        else:
            var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
            x = (x - mean) / torch.sqrt(var + EPS)
        out = []
        for prefix, rows in (("", x[:, :, :n_img]), ("text_" if c["text_norm"] else "", x[:, :, n_img:])):
            rows = rows * norm[prefix + which + "_weight"]
            out.append(rows + norm[prefix + which + "_bias"] if c["norm"] == "layer" else rows)
        x = torch.cat(out, 2)
    return _turned(state, x)


def _codes64(state, y, transposed):
    """As the quantizer defines them: values, scale and quotient are binary32 numbers, halves go to the even code."""
    c = state["case"]
    n, block = _tokens(c), c["block"]
    k = -(-n // block)
    blocks = y.new_zeros((c["B"], c["nh"], k * block, c["d"]))
    for h in range(c["nh"]):
        blocks[:, h, :n] = y[:, h, state["at"][h]]
    blocks = blocks.unflatten(2, (k, block))
    scale = None
    if c["bits"] != 16:
        blocks = blocks.float().double()
        scale = (blocks.abs().flatten(3).max(-1).values / 127).float().double()
        scale[scale == 0] = 1.0
        shared = scale[..., None, None]
        blocks = (blocks / shared).float().double().round() * shared
    if transposed:
        source = torch.empty(block, dtype=torch.long, device=DEV)
        source[_slots(block)] = torch.arange(block, device=DEV)
        blocks = blocks[:, :, :, source].permute(0, 1, 2, 4, 3)
    else:
        blocks = blocks.flatten(2, 3)
    return blocks if scale is None else (blocks, scale)


def exact(case, seed):
    state = prepare(case, seed)
    c = state["case"]
    x = [t.double() for t in state["x"]]
    norm = {name: w.double() for name, w in state["norm"].items()}
    if c["op"] == "rope":
        return _turned(state, x[0], -1.0 if c["inverse"] else 1.0)
    if c["op"] == "norm_rope":
        return [_forward64(state, which, x[i], norm) for i, which in enumerate("qk")]
    if c["op"] == "backward":
        out = {}
        for i, which in enumerate("qk"):
            leaf = x[i].contiguous().requires_grad_()
            mine = {name: w.clone().requires_grad_() for name, w in norm.items() if which + "_" in name}
            grads = torch.autograd.grad(_forward64(state, which, leaf, mine), [leaf, *mine.values()], state["dy"][i].double())
            out["d" + which] = grads[0]
            out.update(zip(mine, grads[1:]))
        return out
    return [_codes64(state, _forward64(state, "q", x[0], norm), False), _codes64(state, _forward64(state, "k", x[1], norm), False),
            _codes64(state, x[2], True)]


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    c = case
    e, size = _elements(c), 2 if c["dtype"] == "bf16" else 4
    table = 4 * (c["d0"] * c["F"] + c["d1"] * c["Hg"] + c["d2"] * c["Wg"])
    padded = c["B"] * c["nh"] * -(-_tokens(c) // c["block"]) * c["block"] * c["d"]
    # a rotation is 6 operations per pair; a norm 2 for the sum of squares and 2 for the weights, 3 more with mean and bias
    turn, norm = 3, {"none": 0, "rms": 4, "layer": 7}[c["norm"]]
    if c["op"] == "rope":
        return {"bytes": 2 * e * size + table, "flops": turn * e}
    if c["op"] == "norm_rope":
        return {"bytes": 2 * 2 * e * size + table, "flops": 2 * e * (turn + norm)}
    if c["op"] == "backward":
        return {"bytes": 2 * 3 * e * size + table, "flops": 2 * e * (turn + 2 * norm + 2)}
    # the values come back as bf16, or as the float32 products of code and scale
    return {"bytes": 3 * e * size + 3 * padded * (2 if c["bits"] == 16 else 4) + table, "flops": 2 * e * (turn + norm) + (0 if c["bits"] == 16 else 3 * 3 * e)}
