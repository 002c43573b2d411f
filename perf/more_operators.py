"""Operators in front of the sub-layer's attention and what it keeps for its backward pass, as named cases with inputs, one
pass, its outputs and what they should be.

Three kinds of case:
  rotary   positions as rotations of pairs of a head's elements, with one axis (text), two (images) or three (video): a
           forward pass, or forward and backward.  The first `rotated` of the heads are turned (queries and keys of a joint
           projection), the others pass
  norm     root-mean-square norm with the residual's addition: a training step, whose norm keeps its input in 16 or 32 bits
           or the normalised row in 8, or a forward pass whose output is held in 8 bits
  linear   a projection whose input is kept in 8 bits for the weight's gradient: a training step, of the projection alone or of
           the norm before it too, which then share what they keep

8 bits: a row goes in groups of 64 elements; a group's scale is the smallest power of two s with max |x| <= 127 s (and at least
2^-126), an element's code rint(x / s), ties to even.

Sizes are those of the configurations of `spion_inputs.py`, of the tests, and in between; `draw` spreads over the same ranges.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 64


def _rotary(name, dtype, B, N, rotated, L, d, sections, ladder="shared", neighbours=False, tokens_first=True, backward=True):
    return dict(name=name, kind="rotary", dtype=dtype, B=B, N=N, rotated=rotated, L=L, d=d, t=sections[0], h=sections[1],
                w=sections[2], ladder=ladder, neighbours=neighbours, tokens_first=tokens_first, backward=backward)


def _norm(name, dtype, rows, D, residual=True, eight="none", backward=True):
    return dict(name=name, kind="norm", dtype=dtype, rows=rows, D=D, residual=residual, eight=eight, backward=backward)


def _linear(name, dtype, rows, M, N, bias=True, normed=False):
    return dict(name=name, kind="linear", dtype=dtype, rows=rows, M=M, N=N, bias=bias, normed=normed)


def listed():
    return [
        # serving: queries and keys of the next token of 64 sequences, three axes; latency
        _rotary("rotary_token_fwd", "bf16", 64, 16, 16, 1, 64, (8, 12, 12), backward=False),
        # configuration 3: queries and keys in the joint projection's output, one axis
        _rotary("rotary_cfg3_step", "bf16", 8, 12, 8, 2048, 64, (32, 0, 0)),
        # a clip of 7 x 11 x 13 patches in fp32, heads before tokens, neighbours paired, a ladder for each axis
        _rotary("rotary_video_f32_step", "f32", 3, 3, 3, 1001, 64, (8, 12, 12), "own", True, False),
        # large images, 128 x 128 patches, two axes, the joint projection of eight heads
        _rotary("rotary_large_step", "bf16", 4, 24, 16, 16384, 64, (0, 16, 16), "own"),
        # serving: the next token of 64 sequences, its normed row in 8 bits
        _norm("norm_token_fwd", "bf16", 64, 512, eight="output", backward=False),
        # the start of the sub-layer at the shape of configuration 3, what it keeps in 8 bits
        _norm("norm_cfg3_step", "bf16", 16384, 256, eight="checkpoint"),
        # full precision, odd sizes
        _norm("norm_odd_f32_step", "f32", 1001, 999, residual=False),
        # a wide model's training step
        _norm("norm_large_step", "bf16", 65536, 4096, eight="checkpoint"),
        # small full-precision training: three heads, an odd number of tokens
        _linear("linear_small_f32_step", "f32", 255, 192, 576),
        # norm and joint projection at the shape of configuration 3
        _linear("linear_cfg3_step", "bf16", 16384, 256, 768, bias=False, normed=True),
        # full-precision training of eight heads
        _linear("linear_f32_step", "f32", 8192, 512, 1536),
        # a wide model's projection over a large batch
        _linear("linear_large_step", "bf16", 65536, 2048, 2048, bias=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A width: mostly a multiple of 64, sometimes any number."""
    n = _log_uniform(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.7 else n


def draw(rng):
    kind = rng.choice(("rotary", "norm", "linear"))
    dtype = rng.choices(("bf16", "f32"), (3, 1))[0]
    backward = rng.random() < 0.7
    if kind == "rotary":
        d = rng.choice((64, 64, 64, 64, 16, 32, 48, 96, 128, 256))
        while True:
            B, N, L = _log_uniform(rng, 1, 64), rng.randint(1, 24), _log_uniform(rng, 1, 16384)
            if B * N * L * d <= 2 ** 26:
                break
        pairs = d // 2
        t = rng.randint(0, pairs)
        h = rng.randint(0, pairs - t)
        w = rng.choice((pairs - t - h, rng.randint(0, pairs - t - h)))
        if t + h + w == 0:
            t = pairs
        return dict(kind=kind, dtype=dtype, B=B, N=N, rotated=rng.randint(1, N), L=L, d=d, t=t, h=h, w=w,
                    ladder=rng.choice(("shared", "own")), neighbours=rng.random() < 0.4, tokens_first=rng.random() < 0.6,
                    backward=backward)
    if kind == "norm":
        while True:
            rows, D = _log_uniform(rng, 1, 65536), _size(rng, 1, 8192)
            if rows * D <= 2 ** 26:
                break
        return dict(kind=kind, dtype=dtype, rows=rows, D=D, residual=rng.random() < 0.7,
                    eight=rng.choice(("none", "checkpoint")) if backward else "output", backward=backward)
    while True:
        rows, M, N = _log_uniform(rng, 1, 65536), _size(rng, 8, 4096), _size(rng, 8, 4096)
        if rows * M * N <= (2 ** 37 if dtype == "bf16" else 2 ** 34) and rows * max(M, N) <= 2 ** 27:
            break
    return dict(kind=kind, dtype=dtype, rows=rows, M=M, N=N, bias=rng.random() < 0.5, normed=rng.random() < 0.4)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
BASE = 10000.0
EPS = 1e-6


def _sections(case):
    return [n for n in (case["t"], case["h"], case["w"]) if n]


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _activations(rows, D, dtype, gen):
    """Rows as a residual stream has them: of different magnitudes, a few columns far larger than the rest."""
    x = torch.randn((rows, D), generator=gen, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device="cuda"))
    x *= torch.where(torch.rand(D, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    return x.to(dtype)


def _positions(case, seed):
    """int64 [axes, L]: text counts on from a place in a long document; patches lie in a grid, row by row, time by time."""
    L, n = case["L"], len(_sections(case))
    start = np.random.default_rng(seed).integers(0, 100000)
    i = np.arange(L)
    if n == 1:
        pos = [start + i]
    else:
        side = max(1, int(round(L ** (1.0 / n))))
        pos = [i // side, i % side] if n == 2 else [start // 100 + i // side ** 2, i // side % side, i % side]
    return torch.from_numpy(np.stack(pos).astype(np.int64)).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "rotary":
        shape = (case["B"], case["L"], case["N"], case["d"])
        if not case["tokens_first"]:
            shape = (case["B"], case["N"], case["L"], case["d"])
        st["x"] = _randn(shape, dtype, gen)
        st["dy"] = _randn(shape, dtype, gen) if case["backward"] else None
        st["positions"] = _positions(case, seed)
        if own:
            import paper_2309_12578_amd as sp
            st["axes"] = sp.rotary_axes(case["d"], _sections(case), base=BASE, ladder=case["ladder"],
                                        neighbours=case["neighbours"], device="cuda")
            st["x"].requires_grad_(case["backward"])
        return st
    rows = case["rows"]
    if case["kind"] == "norm":
        D = case["D"]
        st["x"] = _activations(rows, D, dtype, gen)
        st["residual"] = _activations(rows, D, dtype, gen) if case["residual"] else None
        st["weight"] = (1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(dtype)
        st["dy"] = _randn((rows, D), dtype, gen) if case["backward"] else None
        st["dh"] = _randn((rows, D), dtype, gen) if case["backward"] and case["residual"] else None
        st["inputs"] = [st["x"], st["weight"]] + ([st["residual"]] if case["residual"] else [])
    else:
        M, N = case["M"], case["N"]
        st["x"] = _activations(rows, M, dtype, gen)
        st["w"] = (torch.randn((N, M), generator=gen, device="cuda") / math.sqrt(M)).to(dtype)
        st["b"] = _randn((N,), dtype, gen) if case["bias"] else None
        st["dy"] = _randn((rows, N), dtype, gen)
        st["inputs"] = [st["x"], st["w"]] + ([st["b"]] if case["bias"] else [])
        if case["normed"]:
            st["residual"] = _activations(rows, M, dtype, gen)
            st["weight"] = (1 + 0.2 * torch.randn(M, generator=gen, device="cuda")).to(dtype)
            st["dh"] = _randn((rows, M), dtype, gen)
            st["inputs"] += [st["weight"], st["residual"]]
    if own and case.get("backward", True):
        for t in st["inputs"]:
            t.requires_grad_()
    return st


# ------------------------------------------------------------------------------------------------
# the plain form
# ------------------------------------------------------------------------------------------------
def _eight(x):
    """What the 8 bits of x [rows, D] stand for, in x's type."""
    rows, D = x.shape
    g = torch.nn.functional.pad(x, (0, -D % GROUP)).view(rows, -1, GROUP)
    m, e = torch.frexp(g.abs().amax(dim=2, keepdim=True))
    e = torch.where(m <= 127.0 / 128.0, e - 7, e - 6).clamp(min=-126)
    s = torch.ldexp(torch.ones((), dtype=x.dtype, device=x.device), e)
    return (torch.round(g / s) * s).view(rows, -1)[:, :D]


def _plain_rotary(st):
    case = st["case"]
    d, pairs, sections = case["d"], case["d"] // 2, _sections(case)
    total = sum(sections)
    dev = st["x"].device
    axis = torch.repeat_interleave(torch.arange(len(sections), device=dev), torch.tensor(sections, device=dev))
    n = torch.tensor(sections, device=dev)[axis].double()
    first = (torch.cumsum(torch.tensor(sections, device=dev), 0) - torch.tensor(sections, device=dev))[axis]
    i = torch.arange(total, device=dev)
    exponent = (i - first).double() / n if case["ladder"] == "own" else i.double() / pairs
    # far positions: the angle in 64 bits
    angle = st["positions"][axis].double().t() * torch.pow(BASE, -exponent)
    angle = torch.nn.functional.pad(angle, (0, pairs - total))     # pairs beyond the sections stay
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()  # [L, pairs]
    if case["tokens_first"]:
        cos, sin = cos[:, None], sin[:, None]
    heads = 2 if case["tokens_first"] else 1

    def turn(x, sin):
        some, rest = x.split([case["rotated"], case["N"] - case["rotated"]], dim=heads)
        some = some.float()
        if case["neighbours"]:
            a, b = some[..., 0::2], some[..., 1::2]
            some = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        else:
            a, b = some[..., :pairs], some[..., pairs:]
            some = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        return torch.cat([some.to(x.dtype), rest], dim=heads)

    res = {"y": turn(st["x"], sin)}
    if case["backward"]:
        res["dx"] = turn(st["dy"], -sin)
    return res


def _plain_norm(x, residual, weight, eight):
    """s, 1 / rms, the row as the backward pass has it, y; in 64 bits where codes are chosen: a value next to a border."""
    wide = torch.float64 if eight else torch.float32
    s = x.to(wide)
    if residual is not None:
        s = s + residual.to(wide)
    rstd = 1.0 / torch.sqrt(s.square().mean(dim=1, keepdim=True) + EPS)
    xhat = s * rstd
    kept = _eight(xhat) if eight else xhat
    return s, rstd.float(), kept.float(), xhat * weight.to(wide)


def _plain_norm_grad(dy, dh, weight, rstd, kept):
    g = dy * weight.float()
    dx = rstd * (g - kept * (g * kept).mean(dim=1, keepdim=True))
    if dh is not None:
        dx = dx + dh.float()
    return dx, (dy * kept).sum(dim=0, dtype=torch.float64)


def _plain_norm_case(st):
    case = st["case"]
    dtype = DTYPES[case["dtype"]]
    s, rstd, kept, y = _plain_norm(st["x"], st["residual"], st["weight"], case["eight"] != "none")
    res = {"h": s.to(dtype)} if case["residual"] else {}
    if case["eight"] == "output":
        return {**res, "y": _eight(y).to(torch.bfloat16)}
    res["y"] = y.to(dtype)
    if case["backward"]:
        dx, dw = _plain_norm_grad(st["dy"].float(), st["dh"], st["weight"], rstd, kept)
        res.update(dx=dx.to(dtype), dweight=dw.to(dtype))
    return res


def _plain_linear(st):
    case = st["case"]
    dtype = DTYPES[case["dtype"]]
    w, g = st["w"].float(), st["dy"].float()
    if case["normed"]:
        s, rstd, kept, x = _plain_norm(st["x"], st["residual"], st["weight"], True)
        x, held = x.float(), kept * st["weight"].float()
    else:
        x = st["x"].float()
        held = _eight(x)
    y = torch.matmul(x, w.t())
    if case["bias"]:
        y = y + st["b"].float()
    dx = torch.matmul(g, w)
    res = {"y": y.to(dtype), "dw": torch.matmul(g.t(), held).to(dtype)}
    if case["bias"]:
        res["db"] = g.sum(dim=0, dtype=torch.float64).to(dtype)
    if case["normed"]:
        dx, dweight = _plain_norm_grad(dx, st["dh"], st["weight"], rstd, kept)
        res.update(h=s.to(dtype), dweight=dweight.to(dtype))
    res["dx"] = dx.to(dtype)
    return res


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def _own_rotary(st):
    import paper_2309_12578_amd as sp
    case = st["case"]
    # rotary takes [B, heads, L, d], with any strides
    heads = (lambda t: t.transpose(1, 2)) if case["tokens_first"] else (lambda t: t)
    y = heads(sp.rotary(heads(st["x"]), st["axes"], st["positions"], heads=case["rotated"]))
    if not case["backward"]:
        return {"y": y}
    return {"y": y.detach(), "dx": torch.autograd.grad(y, st["x"], st["dy"])[0]}


def _own_norm(st):
    import paper_2309_12578_amd as sp
    case = st["case"]
    if case["eight"] == "output":
        p, h = sp.rms_norm8(st["x"], st["weight"], st["residual"], EPS)
        y = sp.unpack8(p, torch.bfloat16)
        return {"y": y} if h is None else {"y": y, "h": h}
    y, h, _ = sp.rms_norm(st["x"], st["weight"], st["residual"], EPS, checkpoint=case["eight"] == "checkpoint")
    outputs, grads = ([y, h], [st["dy"], st["dh"]]) if case["residual"] else ([y], [st["dy"]])
    dx, dw = torch.autograd.grad(outputs, st["inputs"], grads)[:2]
    res = {"y": y.detach(), "dx": dx, "dweight": dw}
    if case["residual"]:
        res["h"] = h.detach()
    return res


def _own_linear(st):
    import paper_2309_12578_amd as sp
    case = st["case"]
    if not case["normed"]:
        y = sp.linear8(st["x"], st["w"], st["b"])
        grads = torch.autograd.grad(y, st["inputs"], st["dy"])
        return dict(zip(("y", "dx", "dw", "db"), (y.detach(), *grads)))
    x, h, p = sp.rms_norm(st["x"], st["weight"], st["residual"], EPS, checkpoint=True)
    y = sp.linear8(x, st["w"], st["b"], checkpoint=p)
    grads = torch.autograd.grad([y, h], st["inputs"], [st["dy"], st["dh"]])
    names = ("dx", "dw") + (("db",) if case["bias"] else ()) + ("dweight",)
    return {"y": y.detach(), "h": h.detach(), **dict(zip(names, grads))}


def run(st):
    kind = st["case"]["kind"]
    with torch.set_grad_enabled(own and st["case"].get("backward", True)):
        if own:
            return {"rotary": _own_rotary, "norm": _own_norm, "linear": _own_linear}[kind](st)
        return {"rotary": _plain_rotary, "norm": _plain_norm_case, "linear": _plain_linear}[kind](st)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    eight = 1.0 + 1.0 / GROUP
    if case["kind"] == "rotary":
        n = case["B"] * case["N"] * case["L"] * case["d"]
        return {"bytes": n * size * (4 if case["backward"] else 2), "flops": 3 * n * (2 if case["backward"] else 1)}
    if case["kind"] == "norm":
        n = case["rows"] * case["D"]
        tensors = 2 + 2 * case["residual"]                       # x, residual; y, h
        if case["eight"] == "output":
            return {"bytes": n * ((tensors - 1) * size + 2), "flops": 6 * n}
        # dy, dh; dx; what is kept: written and read where it is not an output or an input itself
        kept = 2 * eight if case["eight"] == "checkpoint" else size
        return {"bytes": n * ((tensors + 2 + case["residual"]) * size + kept), "flops": 14 * n}
    rows, M, N = case["rows"], case["M"], case["N"]
    # x, y; dy, dx; w twice, dw; what is kept, written and read
    values = 2 * rows * M + 2 * rows * N + 3 * M * N + (3 * rows * M if case["normed"] else 0)
    return {"bytes": values * size + 2 * eight * rows * M, "flops": 6 * rows * M * N}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_eight(x):
    rows, D = x.shape
    x = torch.cat([x, torch.zeros((rows, -D % GROUP), dtype=x.dtype, device=x.device)], dim=1)
    top = x.abs().unflatten(1, (-1, GROUP)).max(dim=2).values
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / 127.0)))
    # the logarithm may be off where the quotient is next to a power of two
    scale = torch.where(scale * 127.0 < top, scale * 2.0, scale)
    scale = torch.where(scale * 63.5 >= top, scale / 2.0, scale)
    scale = torch.where(top > 0, scale, torch.ones_like(scale)).clamp(min=2.0 ** -126).repeat_interleave(GROUP, dim=1)
    q = x / scale
    whole = torch.floor(q)
    part = q - whole
    up = (part > 0.5) | ((part == 0.5) & (whole % 2 != 0))
    return ((whole + up.double()) * scale)[:, :D]


def _exact_rotary(case, st):
    d, sections = case["d"], _sections(case)
    which = [a for a, n in enumerate(sections) for _ in range(n)]
    place = [j / n for n in sections for j in range(n)] if case["ladder"] == "own" else [i / (d // 2) for i in range(len(which))]
    rest = d // 2 - len(which)
    freq, which = [BASE ** -p for p in place] + [0.0] * rest, which + [0] * rest
    pos = st["positions"].cpu().double().numpy()
    angle = torch.from_numpy(pos[which].T * np.array(freq)).cuda()   # [L, pairs]
    phase = torch.polar(torch.ones_like(angle), angle)

    def turned(x, phase):
        x = (x.transpose(1, 2) if case["tokens_first"] else x).double()
        pair = x.unflatten(-1, (-1, 2)) if case["neighbours"] else x.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pair[:, :case["rotated"]].contiguous()) * phase)
        z = torch.cat([z, pair[:, case["rotated"]:]], dim=1)
        out = z.flatten(-2) if case["neighbours"] else z.transpose(-1, -2).flatten(-2)
        return out.transpose(1, 2) if case["tokens_first"] else out

    res = {"y": turned(st["x"], phase)}
    if case["backward"]:
        res["dx"] = turned(st["dy"], phase.conj())
    return res


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "rotary":
        return _exact_rotary(case, st)
    x, res = st["x"].double(), {}
    normed = case["kind"] == "norm" or case["normed"]
    if normed:
        weight = st["weight"].double()
        if st["residual"] is not None:
            x = x + st["residual"].double()
            res["h"] = x
        root = torch.sqrt(torch.linalg.vector_norm(x, dim=1, keepdim=True) ** 2 / x.shape[1] + EPS)
        unit = x / root
        if case.get("eight") == "output":
            return {**res, "y": _exact_eight(unit * weight)}
        x = unit * weight
        kept = unit if case.get("eight") == "none" else _exact_eight(unit)
    if case["kind"] == "norm":
        res["y"] = x
        g = st["dy"].double() if case["backward"] else None
    else:
        w, dy = st["w"].double(), st["dy"].double()
        res["y"] = torch.matmul(x, w.t())
        held = kept * weight if normed else _exact_eight(x)
        res["dw"] = torch.matmul(dy.t(), held)
        if case["bias"]:
            res["y"] += st["b"].double()
            res["db"] = dy.sum(0)
        g = torch.matmul(dy, w)
    if g is not None and normed:
        res["dweight"] = (g * kept).sum(0)
        gw = g * weight
        g = (gw - kept * ((gw * kept).sum(1, keepdim=True) / x.shape[1])) / root
        if st["dh"] is not None:
            g = g + st["dh"].double()
    if g is not None:
        res["dx"] = g
    return res
