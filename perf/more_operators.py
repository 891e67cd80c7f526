"""What is timed of the library's operators on 8-bit floats with block scales, root-mean-square norms and orthogonalised updates.

"norm": the root-mean-square norm of a block's input with the residual's addition, into its own type or into 8-bit floats with a scale per
128 elements, as the next product reads it (and its gradient's product the transpose's form); with ``grad`` also the way back.
"quantise": a tensor to 8-bit floats with a scale per 128 elements of a row, or per 128 x 128 elements (``square``), and back.
"product": a product of two tensors held that way (rows of both against each other), as a linear layer or its gradients take it.
"orthogonalise": the update of one layer, or of a stack of like ones, brought near the orthogonal matrix next to it by Newton-Schulz products.

The plain forms are the same formulas in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

_NONE = dict(op="", rows=0, cols=0, m=0, n=0, k=0, batch=0, dtype="bf16", weight="same", forms="none", kind="e4m3", kind_b="e4m3", add=False, grad=False,
             square=False, steps=0)


def _case(**kw):
    return dict(_NONE, **kw)


def listed():
    return [
        # one token at the entry of a feed-forward layer: launch and host time are all there is
        _case(name="norm-token", op="norm", rows=1, cols=1600, add=True, forms="rows"),
        # a training step's tokens at the same place: what the layer's product and its weight's gradient read
        _case(name="norm-train", op="norm", rows=8192, cols=1600, add=True, forms="both"),
        # the norm of a layer whose product stays in 16 bits, forward and backward, the residual's gradient joined
        _case(name="norm-grad", op="norm", rows=8192, cols=1600, add=True, grad=True),
        # the largest: fp32 activations of odd width, forward and backward
        _case(name="norm-odd-fp32", op="norm", rows=30011, cols=1301, dtype="fp32", grad=True),
        # a weight once per step: both products of a step read the same rounded values
        _case(name="quantise-weight", op="quantise", rows=6400, cols=1600, dtype="fp32", forms="both", square=True),
        # the gradient of a layer's output, in the type of wider range
        _case(name="quantise-gradient", op="quantise", rows=8192, cols=6400, forms="both", kind="e5m2"),
        # one token through a feed-forward layer
        _case(name="product-token", op="product", m=1, n=6400, k=1600),
        # sizes that are multiples of nothing, a gradient against a weight
        _case(name="product-odd", op="product", m=1111, n=2601, k=651, dtype="fp32", kind="e5m2"),
        # a training batch through a feed-forward layer
        _case(name="product-train", op="product", m=8192, n=6400, k=1600),
        # the only layer of the smallest workload
        _case(name="orthogonalise-tiny", op="orthogonalise", batch=1, rows=256, cols=512, steps=5, dtype="fp32"),
        # an attention layer's projection of a GPT-2-XL list
        _case(name="orthogonalise-layer", op="orthogonalise", batch=1, rows=1600, cols=1600, steps=5),
        # both feed-forward weights of two layers, stored as out x in
        _case(name="orthogonalise-stack", op="orthogonalise", batch=2, rows=6400, cols=1600, steps=5),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _matrix(rng, most):
    """Rows and columns of at most `most` elements: widths of models in one half, anything in the other."""
    rows = _spread(rng, 1, 60000)
    cols = min(_spread(rng, 1, 8192), max(1, most // rows))
    if cols > 64 and rng.random() < 0.5:
        cols = cols // 64 * 64
    return rows, cols


def draw(rng):
    op = rng.choice(["norm", "norm", "quantise", "product", "orthogonalise"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    kind = rng.choice(["e4m3", "e4m3", "e5m2"])
    if op == "norm":
        rows, cols = _matrix(rng, 13_000_000)
        return _case(op=op, rows=rows, cols=cols, dtype=dtype, weight=rng.choice(["same", "fp32"]), add=rng.random() < 0.5,
                     forms=rng.choice(["none", "rows", "cols", "both"]), kind=kind, grad=rng.random() < 0.5)
    if op == "quantise":
        rows, cols = _matrix(rng, 40_000_000)
        return _case(op=op, rows=rows, cols=cols, dtype=dtype, forms=rng.choice(["rows", "cols", "both"]), kind=kind, square=rng.random() < 0.3)
    if op == "product":
        m = _spread(rng, 1, 8192)
        n, k = _spread(rng, 64, 6400), _spread(rng, 32, 1600)
        if rng.random() < 0.5:
            n, k = max(64, n // 64 * 64), max(32, k // 32 * 32)
        return _case(op=op, m=m, n=n, k=k, dtype=dtype, kind=kind, kind_b=rng.choice(["e4m3", "e4m3", "e5m2"]))
    rows, cols = _spread(rng, 2, 4000), _spread(rng, 2, 4000)
    if rng.random() < 0.5:
        rows, cols = max(2, rows // 32 * 32), max(2, cols // 32 * 32)
    steps = rng.choice([5, 5, 3, 6])
    low, high = min(rows, cols), max(rows, cols)
    most = int(7e11 / (steps * (4 * low * low * high + 2 * low ** 3)))
    return _case(op=op, batch=max(1, min(_spread(rng, 1, 24), most, 20_000_000 // (rows * cols))), rows=rows, cols=cols if most else min(cols, 2000), steps=steps, dtype=dtype)


# ------------------------------------------------------------------ inputs

_DTYPES = dict(bf16=torch.bfloat16, fp16=torch.float16, fp32=torch.float32)
_EPS = 1e-5
_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _activations(rows, cols, dtype, gen, scale=1.0):
    """Normal values whose columns differ in size, as a layer's outputs do."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x *= torch.exp2(torch.randn(1, cols, generator=gen, device="cuda")) * scale
    return x.to(dtype)


def _update(batch, rows, cols, dtype, gen):
    """A momentum as layers have it: a part of low rank that carries most of it, and noise in all directions."""
    rank = max(1, min(rows, cols) // 8)
    a = torch.randn(batch, rows, rank, generator=gen, device="cuda") * torch.exp2(torch.randn(batch, 1, rank, generator=gen, device="cuda"))
    x = a @ torch.randn(batch, rank, cols, generator=gen, device="cuda") / math.sqrt(rank)
    return ((x + 0.3 * torch.randn(batch, rows, cols, generator=gen, device="cuda")) * 1e-3).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case, seed=seed)
    dtype = _DTYPES[case["dtype"]]
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "norm":
        w = 1.0 + 0.3 * torch.randn(cols, generator=gen, device="cuda")
        state.update(x=_activations(rows, cols, dtype, gen), r=_activations(rows, cols, dtype, gen) if case["add"] else None,
                     w=w if case["weight"] == "fp32" else w.to(dtype))
        if case["grad"]:
            state.update(dy=_activations(rows, cols, dtype, gen, scale=1e-3), dh=_activations(rows, cols, dtype, gen, scale=1e-3) if case["add"] else None)
    elif case["op"] == "quantise":
        state.update(x=_activations(rows, cols, dtype, gen))
    elif case["op"] == "product":   # both sides as a quantisation before this pass left them
        state.update(a=_hold(_activations(case["m"], case["k"], torch.float32, gen), case["kind"]),
                     b=_hold(torch.randn(case["n"], case["k"], generator=gen, device="cuda") * 0.02, case["kind_b"]))
    else:
        state.update(x=_update(case["batch"], rows, cols, dtype, gen))
    return state


# ------------------------------------------------------------------ plain forms

_BITS = dict(e4m3=(3, -6, 9), e5m2=(2, -14, 16))   # of the mantissa; the least normal exponent; the largest value is 0.875 times two to this
_FLOAT8 = dict(e4m3=torch.float8_e4m3fn, e5m2=torch.float8_e5m2)


def _tiles(x, high):
    """x, padded, as blocks of high x 128: (row blocks, high, column blocks, 128)."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 128, 0, -rows % high))
    return x.view(-1, high, x.shape[1] // 128, 128)


def _scaled(x, kind, high):
    """Blocks of x over their scale 2^e, the least that leaves no element above the type's largest, and e (in 64 bits: values lie next to borders)."""
    b = _tiles(x, high)
    m, e = torch.frexp(b.abs().amax((1, 3), keepdim=True))
    top = _BITS[kind][2]
    e = torch.where(m <= 0.875, e - top, e - top + 1).clamp(min=-127)
    return b.double() * torch.exp2(-e.double()), e


def _rounded(v, kind):
    """To the type's values, to nearest even."""
    mantissa, least, _ = _BITS[kind]
    step = torch.exp2((torch.frexp(v.abs()).exponent - 1).clamp(min=least).double() - mantissa)
    return torch.round(v / step) * step


def _represented(x, kind, high=1):
    """The values that x's 8-bit form stands for; they are exact in bf16."""
    v, e = _scaled(x, kind, high)
    return (_rounded(v, kind) * torch.exp2(e.double())).view(-1, v.shape[2] * 128)[:x.shape[0], :x.shape[1]].bfloat16()


def _forms(x, forms, kind, square):
    high = 128 if square else 1
    out = {}
    if forms in ("rows", "both"):
        out["rows"] = _represented(x, kind, high)
    if forms in ("cols", "both"):
        out["cols"] = _represented(x.t().contiguous(), kind, high)
    return out


def _hold(x, kind):
    """x's 8-bit form as a user holds it: rows padded to 128 bytes; scales in tiles of 128 rows by 4 blocks."""
    v, e = _scaled(x, kind, 1)
    codes = _rounded(v, kind).float().to(_FLOAT8[kind]).view(torch.uint8).view(-1, v.shape[2] * 128)
    s = (e.view(v.shape[0], -1) + 127).to(torch.uint8)
    s = torch.nn.functional.pad(s, (0, -s.shape[1] % 4, 0, -s.shape[0] % 128))
    scales = s.view(s.shape[0] // 128, 4, 32, -1, 4).permute(0, 3, 2, 1, 4).reshape(-1).contiguous()
    return dict(rows=x.shape[0], cols=x.shape[1], kind=kind, codes=codes.contiguous(), scales=scales)


def _values(h):
    rows, cols = h["rows"], h["cols"]
    v = h["codes"].view(_FLOAT8[h["kind"]]).float()
    s = h["scales"].view(-(-rows // 128), -1, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-(-rows // 128) * 128, -1)[:rows, :v.shape[1] // 128]
    return (v.unflatten(1, (-1, 128)) * torch.exp2(s.float() - 127.0).unsqueeze(-1)).flatten(1)[:, :cols]


def _plain_norm(state):
    dtype = state["x"].dtype
    h = state["x"] if state["r"] is None else (state["x"].float() + state["r"].float()).to(dtype)
    wide = h.double()
    r = torch.rsqrt(wide.square().mean(1, keepdim=True) + _EPS)
    out = dict(rstd=r.squeeze(1).float())   # (y is formed with it as it is stored)
    if state["r"] is not None:
        out["h"] = h
    y = wide * out["rstd"].double().unsqueeze(1) * state["w"].double()
    if state["forms"] == "none":
        out["y"] = y.to(dtype)
    else:
        out.update(_forms(y, state["forms"], state["kind"], False))
    if state["grad"]:
        n = h.float() * out["rstd"].unsqueeze(1)
        dy = state["dy"].float()
        g = dy * state["w"].float()
        dh = out["rstd"].unsqueeze(1) * (g - n * (g * n).mean(1, keepdim=True))
        out["dx"] = (dh if state["dh"] is None else dh + state["dh"].float()).to(dtype)
        out["dw"] = (dy.double() * n).sum(0).float()
    return out


def _plain_orthogonalise(x, steps):
    a, b, c = _COEFFICIENTS
    dtype = torch.bfloat16 if x.dtype == torch.float32 else x.dtype
    x = x.float()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = x / x.double().square().sum((1, 2), keepdim=True).sqrt().float()
    for _ in range(steps):
        g = x @ x.transpose(1, 2)
        x = a * x + (b * g + c * (g @ g)) @ x
    return (x.transpose(1, 2) if tall else x).to(dtype).contiguous()


def _plain(state):
    op, dtype = state["op"], _DTYPES[state["dtype"]]
    if op == "norm":
        return _plain_norm(state)
    if op == "quantise":
        return _forms(state["x"].float(), state["forms"], state["kind"], state["square"])
    if op == "product":
        return dict(out=(_values(state["a"]) @ _values(state["b"]).t()).to(dtype))
    return dict(out=_plain_orthogonalise(state["x"], state["steps"]))


# ------------------------------------------------------------------ the library's calls

def _own_values(made, forms):
    from paper_2312_08538_b200 import binding as cb
    named = zip(("rows", "cols"), made) if forms == "both" else ((forms, made),)
    return {name: cb.f8_dequantise(form, dtype=torch.bfloat16) for name, form in named}


def _own(state):
    from paper_2312_08538_b200 import binding as cb
    op, dtype = state["op"], _DTYPES[state["dtype"]]
    if op == "norm":
        forms = None if state["forms"] == "none" else state["forms"]
        y, h, rstd = cb.rms_norm(state["x"], state["w"], _EPS, add=state["r"], forms=forms, kind=state["kind"])
        out = dict(rstd=rstd)
        if state["r"] is not None:
            out["h"] = h
        if forms is None:
            out["y"] = y
        else:
            out.update(_own_values(y, forms))
        if state["grad"]:
            out["dx"], out["dw"] = cb.rms_norm_grad(state["dy"], h, state["w"], rstd, add=state["dh"])
        return out
    if op == "quantise":
        return _own_values(cb.f8_quantise(state["x"], forms=state["forms"], kind=state["kind"], square=state["square"]), state["forms"])
    if op == "product":
        a, b = (cb.F8(h["rows"], h["cols"], h["kind"], h["codes"], h["scales"]) for h in (state["a"], state["b"]))
        return dict(out=cb.f8_matmul(a, b, dtype=dtype))
    return dict(out=cb.orthogonalise(state["x"], steps=state["steps"], coefficients=_COEFFICIENTS))


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    held = 1.0 + 1.0 / 128
    d = case["rows"] * case["cols"]
    n_forms = dict(none=0, rows=1, cols=1, both=2)[case["forms"]]
    shown = n_forms * (2 * held + 2)   # a form out and in again, its values out
    if case["op"] == "norm":   # x and the residual in, their sum out; the gradients in, x's gradient out
        one = size * (1 + 2 * case["add"] + (n_forms == 0)) + shown + case["grad"] * size * (2 + case["add"])
        if case["grad"]:
            one += 0 if case["add"] else size
        return dict(bytes=d * one + 4 * case["rows"] + 4 * case["cols"], flops=d * (5 + case["add"] + 9 * case["grad"]))
    if case["op"] == "quantise":
        return dict(bytes=d * (size + shown), flops=3 * d * n_forms)
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return dict(bytes=held * k * (m + n) + size * m * n, flops=2 * m * n * k)
    low, high = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])   # (products of a matrix with its transpose are symmetric)
    return dict(bytes=case["batch"] * d * (size + 2), flops=case["batch"] * case["steps"] * (3 * low * low * high + low ** 3))


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_grid(kind):
    """The values from zero up of an 8-bit type, in order, from the meaning of its codes."""
    mantissa = dict(e4m3=3, e5m2=2)[kind]
    bias = dict(e4m3=7, e5m2=15)[kind]
    most = dict(e4m3=448.0, e5m2=57344.0)[kind]
    grid = []
    for code in range(128):
        exponent, part = code >> mantissa, (code & ((1 << mantissa) - 1)) / (1 << mantissa)
        grid.append(math.ldexp(1.0 + part, exponent - bias) if exponent else math.ldexp(part, 1 - bias))
    return torch.tensor([g for g in grid if g <= most], dtype=torch.float64, device="cuda")


def _exact_form(x, kind, high):
    """x in 64 bits; what its form stands for."""
    rows, cols = x.shape
    grid = _exact_grid(kind)
    across, down = -(-cols // 128), -(-rows // high)
    big = torch.zeros(down * high, across * 128, dtype=torch.float64, device="cuda")
    big[:rows, :cols] = x
    most = big.abs().view(down, high, across, 128).permute(0, 2, 1, 3).reshape(down, across, -1).max(-1).values
    power = torch.zeros_like(most)
    power[most > 0] = torch.ceil(torch.log2(most[most > 0] / grid[-1]))
    power = torch.where(most > grid[-1] * torch.exp2(power), power + 1, power)   # (the logarithm is rounded)
    power = torch.where((most > 0) & (most <= grid[-1] * torch.exp2(power - 1)), power - 1, power)
    scale = torch.exp2(torch.where(most > 0, power, -127.0).clamp(min=-127.0)).repeat_interleave(high, 0).repeat_interleave(128, 1)[:rows, :cols]
    size = x.abs() / scale
    below = (torch.searchsorted(grid, size, right=True) - 1).clamp(0, grid.numel() - 2)
    part = (size - grid[below]) - (grid[below + 1] - size)
    return torch.copysign(grid[below + ((part > 0) | ((part == 0) & (below % 2 == 1))).long()] * scale, x)


def _exact_forms(x, case, high):
    out = {}
    if case["forms"] in ("rows", "both"):
        out["rows"] = _exact_form(x, case["kind"], high)
    if case["forms"] in ("cols", "both"):
        out["cols"] = _exact_form(x.t().contiguous(), case["kind"], high)
    return out


def _exact_norm(case, state):
    x = state["x"]
    h = x if state["r"] is None else (x.float() + state["r"].float()).to(x.dtype)   # (rounded to its type by definition)
    v, w = h.double(), state["w"].double()
    mean = torch.einsum("rc,rc->r", v, v) / case["cols"]
    root = 1.0 / torch.sqrt(mean + _EPS)
    out = dict(rstd=root)
    if state["r"] is not None:
        out["h"] = h.double()
    y = torch.einsum("rc,r,c->rc", v, root.float().double(), w)   # (with the root as it is stored, by definition)
    if case["forms"] == "none":
        out["y"] = y
    else:
        out.update(_exact_forms(y, case, 1))
    if case["grad"]:
        dy = state["dy"].double()
        # y_j = h_j root w_j with d root / d h_i = -root^3 h_i / cols
        along = torch.einsum("rc,rc,c->r", dy, v, w) * root ** 3 / case["cols"]
        dh = dy * w * root[:, None] - v * along[:, None]
        out["dx"] = dh if state["dh"] is None else dh + state["dh"].double()
        out["dw"] = torch.einsum("rc,rc,r->c", dy, v, root)
    return out


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        return _exact_norm(case, state)
    if op == "quantise":
        return _exact_forms(state["x"].double(), case, 128 if case["square"] else 1)
    if op == "product":
        sides = []
        for h in (state["a"], state["b"]):
            rows, cols, codes = h["rows"], h["cols"], h["codes"].cpu().numpy().reshape(h["rows"], -1)
            r, c = np.arange(rows)[:, None], np.arange(codes.shape[1] // 128)[None, :]
            tiles = (cols + 511) // 512
            at = ((r // 128) * tiles + c // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + c % 4
            power = np.repeat(h["scales"].cpu().numpy()[at].astype(np.int64) - 127, 128, 1)
            grid = _exact_grid(h["kind"]).cpu().numpy()
            values = np.where(codes & 128, -1.0, 1.0) * grid[np.minimum(codes & 127, grid.size - 1)]
            sides.append(torch.from_numpy(np.ldexp(values, power)[:, :cols]).cuda())
        return dict(out=sides[0] @ sides[1].t())
    # U f(S) V^T for X = U S V^T, f one step's polynomial as often as there are steps, by the same products in 64 bits: of the shorter
    # side's Gram matrix and a factor in front of X
    a, b, c = _COEFFICIENTS
    out = []
    for x in state["x"].double():
        flip = x.shape[0] > x.shape[1]
        y = x.t() if flip else x
        y = y / torch.linalg.vector_norm(y)
        for _ in range(case["steps"]):
            g = y @ y.t()
            front = c * g
            front.diagonal().add_(b)
            front = front @ g
            front.diagonal().add_(a)
            y = front @ y
        out.append(y.t() if flip else y)
    return dict(out=torch.stack(out))
