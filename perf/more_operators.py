"""The operators around attention in a transformer over the rows of a sparse tensor, as cases that can be timed and compared.

Kinds of pass
  rope   rotary positions of query and key heads, every axis (a token's place, or a voxel's x, y, z, a frame's time, height, width)
         turning a part of the head; in training the gradient too
  norm   root-mean-square norm with the residual's addition: forward, then the gradients of rows and weight
  serve  the same norm with its output in 8 bits (a power of two as the scale of each 128 elements of a row), and the product of
         these rows with weights that are kept in 8 bits, in bf16
  q8     rows to 8 bits and their product with 8-bit weights; in training also both gradients as products of operands in 8 bits
  ffn    gated feed-forward block: y = (act(x Wg^T) * (x Wu^T)) Wo^T; in training also the gradients of rows and weights

With `own` false a pass computes the operators in their plain form: products, sums, exponentials and indexing in 32 bits (angles
in 64), rounded once at the end.  With `own` true it makes the calls of paper_2012_13846_amd.binding.
"""
import math

import torch

own = False


# ---- the cases -------------------------------------------------------------------------------------------------
def _rope(n, heads, kv_heads, dim, parts, far, split, dtype, train):
    """parts: elements of a head that each axis turns, as a text; far: positions lie in 0 .. far - 1 (voxels: around 0)."""
    return {"kind": "rope", "n": n, "heads": heads, "kv_heads": kv_heads, "dim": dim, "parts": ",".join(str(p) for p in parts), "far": far,
            "split": split, "dtype": dtype, "train": train}


def _norm(n, c, residual, dtype):
    return {"kind": "norm", "n": n, "c": c, "residual": residual, "dtype": dtype}


def _serve(n, c, m, dtype):
    return {"kind": "serve", "n": n, "c": c, "m": m, "dtype": dtype}


def _q8(n, c, m, dtype, train):
    return {"kind": "q8", "n": n, "c": c, "m": m, "dtype": dtype, "train": train}


def _ffn(n, c, m, act, dtype, train):
    return {"kind": "ffn", "n": n, "c": c, "m": m, "act": act, "dtype": dtype, "train": train}


def listed():
    return [
        # a serving batch's next tokens, far into their sessions: launches and latency
        {"name": "rope_b96_h32kv8_d128_bf16", **_rope(96, 32, 8, 128, [128], 200000, True, "bf16", False)},
        # training on the rows of four fine clouds, positions from voxel coordinates
        {"name": "rope_batch4_xyz_d32_bf16", **_rope(373601, 8, 8, 32, [12, 10, 10], 512, False, "bf16", True)},
        # one object at the coarsest grid: launches and latency
        {"name": "norm_one_shape_c128_bf16", **_norm(1428, 128, True, "bf16")},
        # a width that is no whole number of 16-byte pieces, without a residual
        {"name": "norm_odd_c77_f32", **_norm(70001, 77, False, "f32")},
        # training a token model with wide rows
        {"name": "norm_wide_c4096_bf16", **_norm(16384, 4096, True, "bf16")},
        # one user's next token: weights are read once
        {"name": "serve_b1_c4096_m6144_bf16", **_serve(1, 4096, 6144, "bf16")},
        # reading a batch of prompts
        {"name": "serve_prompt_c4096_m6144_bf16", **_serve(16384, 4096, 6144, "bf16")},
        # a narrow odd layer over the voxels of one cloud
        {"name": "q8_odd_c200_m77_f32", **_q8(70001, 200, 77, "f32", False)},
        # a projection of a token model trained in 8 bits
        {"name": "q8_train_c2048_bf16", **_q8(8192, 2048, 2048, "bf16", True)},
        # a small serving batch's next tokens: weights are read once
        {"name": "ffn_b8_c4096_m8192_bf16", **_ffn(8, 4096, 8192, "silu", "bf16", False)},
        # training on the voxels of one fine cloud, full precision, odd widths
        {"name": "ffn_odd_c100_m270_f32", **_ffn(20011, 100, 270, "gelu", "f32", True)},
        # training a token model
        {"name": "ffn_train_c2048_m8192_bf16", **_ffn(8192, 2048, 8192, "silu", "bf16", True)},
    ]


def draw(rng):
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):
        return rng.choice([span(lo, hi), 8 * span(max(1, lo // 8), hi // 8), 2 ** rng.randint(max(4, lo.bit_length() - 1), hi.bit_length() - 1)])

    kind = rng.choice(["rope", "norm", "serve", "q8", "ffn", "ffn"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "rope":
        dim = rng.choice([16, 32, 64, 64, 80, 96, 128, 128, rng.randint(2, 128)])
        axes = rng.choice([1, 1, 2, 3, 3, 4])
        left, parts = dim // 2, []
        for a in range(axes):
            parts.append(2 * (left // (axes - a) if rng.random() < 0.7 else rng.randint(0, left)))
            left -= parts[-1] // 2
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4])
        n = span(1, max(2, min(400000, 150_000_000 // ((heads + kv) * dim))))
        return _rope(n, heads, kv, dim, parts, span(2, 200000), rng.random() < 0.5, dtype, rng.random() < 0.6)
    if kind == "norm":
        c = width(16, 8192)
        return _norm(span(1, min(400000, 40_000_000 // c)), c, rng.random() < 0.7, dtype)
    c, m = width(16, 8192), width(16, 8192)
    if kind in ("serve", "q8"):
        most = 200_000_000_000 // (c * m)
        n = span(1, max(2, min(50000, most, 40_000_000 // max(c, m))))
        return _serve(n, c, m, dtype) if kind == "serve" else _q8(n, c, m, dtype, n >= 16 and rng.random() < 0.4)
    most = (100_000_000_000 if dtype == "bf16" else 12_000_000_000) // (c * m)
    train = rng.random() < 0.6
    return _ffn(span(1, max(2, min(50000, most, 40_000_000 // max(c, m)))), c, m, rng.choice(["silu", "silu", "gelu"]), dtype, train)


# ---- what a program holds before the call ----------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _parts(case):
    return [int(p) for p in case["parts"].split(",")]


def _to_q8(x):
    """Rows x [n][c] in 8 bits: codes [n][128 * blocks] (zeros behind c) and one power of two for each 128 elements of a row,
    [n][blocks rounded up to 4] (1 in the places behind): the least that leaves no element beyond 448."""
    n, c = x.shape
    blocks = (c + 127) // 128
    v = torch.zeros((n, blocks * 128), device=x.device)
    v[:, :c] = x
    v = v.view(n, blocks, 128)
    m, e = torch.frexp(v.abs().amax(2))                       # top = m * 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m > 0, e - 9 + (m > 0.875).int(), 0).clamp_(-127, 127)
    codes = torch.ldexp(v, -e[:, :, None]).to(torch.float8_e4m3fn).view(n, blocks * 128)
    scales = torch.full((n, (blocks + 3) // 4 * 4), 127, dtype=torch.uint8, device=x.device)
    scales[:, :blocks] = (e + 127).to(torch.uint8)
    return codes, scales.view(torch.float8_e8m0fnu)


def _from_q8(q, c):
    """The values of the first c elements of every row, in 32 bits."""
    codes, scales = q
    n, wide = codes.shape
    e = scales.view(torch.uint8)[:, :wide // 128].int() - 127
    return torch.ldexp(codes.float().view(n, wide // 128, 128), e[:, :, None]).view(n, wide)[:, :c]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    s = {"case": case}
    n = case["n"]
    if case["kind"] == "rope":
        heads, kv, dim, axes = case["heads"], case["kv_heads"], case["dim"], len(_parts(case))
        w = normal(n, heads + 2 * kv, dim).to(dt)
        s["x"] = w[:, :heads + kv]                            # the queries and keys of a fused projection
        if case["train"]:
            s["dy"] = normal(n, heads + kv, dim).to(dt)
        if axes == 3:                                         # columns 1 .. 3 of a sparse tensor's coordinates, which lie around 0
            coords = torch.randint(-(case["far"] // 2), case["far"] - case["far"] // 2, (n, 4), dtype=torch.int32, device="cuda", generator=g)
            s["pos"] = coords[:, 1:]
        else:
            s["pos"] = torch.randint(0, case["far"], (n, axes), dtype=torch.int32, device="cuda", generator=g)
        return s
    c = case["c"]
    s["x"] = (1.5 * normal(n, c) * (0.5 + torch.rand((n, 1), device="cuda", generator=g))).to(dt)   # rows of unlike size
    if case["kind"] in ("norm", "serve"):
        s["gamma"] = 1 + 0.2 * normal(c)
        s["res"] = normal(n, c).to(dt) if case.get("residual", True) else None
    if case["kind"] == "norm":
        s["dy"] = normal(n, c).to(dt)
        s["dh"] = normal(n, c).to(dt) if case["residual"] else None
        return s
    m = case["m"]
    if case["kind"] == "serve":
        s["w"] = _to_q8(normal(m, c) / math.sqrt(c))          # laid out once
    elif case["kind"] == "q8":
        w = (normal(m, c) / math.sqrt(c)).to(dt)
        if case["train"]:
            s["w"], s["dy"] = w, normal(n, m).to(dt)          # weights change with every step
        else:
            s["w"] = _to_q8(w)
    else:
        s["w_in"], s["w_out"] = (normal(2 * m, c) / math.sqrt(c)).to(dt), (normal(c, m) / math.sqrt(m)).to(dt)
        if case["train"]:
            s["dy"] = normal(n, c).to(dt)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------
def _run_own(s):
    from paper_2012_13846_amd import binding as sp
    case = s["case"]
    if case["kind"] == "rope":
        turn = dict(parts=_parts(case), base=10000.0, split=case["split"])
        out = {"y": sp.sp_rope_fwd(s["x"], s["pos"], **turn)}
        if case["train"]:
            out["dx"] = sp.sp_rope_bwd(s["dy"], s["pos"], **turn)
        return out
    if case["kind"] == "norm":
        h, y, rstd = sp.sp_rms_norm_fwd(s["x"], s["gamma"], residual=s["res"], eps=1e-5)
        dx, dgamma = sp.sp_rms_norm_bwd(h, s["dy"], s["gamma"], rstd, dh=s["dh"])
        return {"h": h, "y": y, "rstd": rstd, "dx": dx, "dgamma": dgamma}
    if case["kind"] == "serve":
        h, q = sp.sp_rms_norm_q8(s["x"], s["gamma"], residual=s["res"], eps=1e-5)
        return {"h": h, "y": sp.sp_q8_linear(q, s["w"], torch.bfloat16)}
    if case["kind"] == "q8":
        x, dt = s["x"], s["x"].dtype
        if not case["train"]:
            return {"y": sp.sp_q8_linear(sp.sp_q8_rows(x), s["w"], dt)}
        w, dy = s["w"], s["dy"]
        y = sp.sp_q8_linear(sp.sp_q8_rows(x), sp.sp_q8_rows(w), dt)
        dx = sp.sp_q8_linear(sp.sp_q8_rows(dy), sp.sp_q8_rows(w, transposed=True), dt)
        dw = sp.sp_q8_linear(sp.sp_q8_rows(dy, transposed=True), sp.sp_q8_rows(x, transposed=True), dt)
        return {"y": y, "dx": dx, "dw": dw}
    if not case["train"]:
        return {"y": sp.sp_ffn_fwd(s["x"], s["w_in"], s["w_out"], act=case["act"], keep=False)}
    y, gu = sp.sp_ffn_fwd(s["x"], s["w_in"], s["w_out"], act=case["act"], keep=True)
    dx, dw_in, dw_out = sp.sp_ffn_bwd(s["x"], s["w_in"], s["w_out"], gu, s["dy"], act=case["act"])
    return {"y": y, "dx": dx, "dw_in": dw_in, "dw_out": dw_out}


def run(s):
    if own:
        return _run_own(s)
    return {"rope": _plain_rope, "norm": _plain_norm, "serve": _plain_serve, "q8": _plain_q8, "ffn": _plain_ffn}[s["case"]["kind"]](s)


def _pairs(case):
    """First and second element of every pair of a head, its axis and its frequency."""
    first, second, axis, freq, at = [], [], [], [], 0
    for a, part in enumerate(_parts(case)):
        for i in range(part // 2):
            first.append(at + (i if case["split"] else 2 * i))
            second.append(at + (i + part // 2 if case["split"] else 2 * i + 1))
            axis.append(a)
            freq.append(10000.0 ** (-2.0 * i / part))
        at += part
    return first, second, axis, freq


def _plain_rope(s):
    first, second, axis, freq = _pairs(s["case"])
    angle = s["pos"][:, axis].double() * torch.tensor(freq, dtype=torch.float64, device="cuda")
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turned(x, sin):
        y = x.float()
        a, b = y[:, :, first], y[:, :, second]
        y = y.clone()
        y[:, :, first], y[:, :, second] = a * cos - b * sin, a * sin + b * cos
        return y.to(x.dtype)

    out = {"y": turned(s["x"], sin)}
    if s["case"]["train"]:
        out["dx"] = turned(s["dy"], -sin)
    return out


def _summed(s):
    """The residual stream as it is stored."""
    return s["x"] if s["res"] is None else (s["x"].float() + s["res"].float()).to(s["x"].dtype)


def _plain_norm(s):
    dt, c = s["x"].dtype, s["x"].shape[1]
    h = _summed(s)
    f, dy = h.float(), s["dy"].float()
    rstd = 1 / torch.sqrt((f * f).sum(1, keepdim=True) / c + 1e-5)
    hat = f * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - hat * ((g * hat).sum(1, keepdim=True) / c))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"h": h, "y": (hat * s["gamma"]).to(dt), "rstd": rstd[:, 0], "dx": dx.to(dt), "dgamma": (dy * hat).sum(0)}


def _plain_serve(s):
    h, c = _summed(s), s["x"].shape[1]
    f = h.float()
    y = f * (1 / torch.sqrt((f * f).sum(1, keepdim=True) / c + 1e-5)) * s["gamma"]
    return {"h": h, "y": torch.matmul(_from_q8(_to_q8(y), c), _from_q8(s["w"], c).t()).to(torch.bfloat16)}


def _plain_q8(s):
    x, dt = s["x"], s["x"].dtype
    n, c = x.shape

    def rounded(t):
        return _from_q8(_to_q8(t.float()), t.shape[1])

    if not s["case"]["train"]:
        return {"y": torch.matmul(rounded(x), _from_q8(s["w"], c).t()).to(dt)}
    w, dy = s["w"], s["dy"]
    return {"y": torch.matmul(rounded(x), rounded(w).t()).to(dt), "dx": torch.matmul(rounded(dy), rounded(w.t()).t()).to(dt),
            "dw": torch.matmul(rounded(dy.t()), rounded(x.t()).t()).to(dt)}


def _plain_ffn(s):
    case, dt = s["case"], s["x"].dtype
    m = case["m"]
    x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
    gu = torch.matmul(x, w_in.t())
    g, u = gu[:, :m], gu[:, m:]
    if case["act"] == "silu":
        p = 1 / (1 + torch.exp(-g))
        a, da = g * p, p * (1 + g * (1 - p))
    else:
        p = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
        a, da = g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    h = a * u
    out = {"y": torch.matmul(h, w_out.t()).to(dt)}
    if case["train"]:
        dy = s["dy"].float()
        dh = torch.matmul(dy, w_out)
        dgu = torch.cat([dh * u * da, dh * a], 1)
        out.update(dx=torch.matmul(dgu, w_in).to(dt), dw_in=torch.matmul(dgu.t(), x).to(dt), dw_out=torch.matmul(dy.t(), h).to(dt))
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    n = float(case["n"])
    if case["kind"] == "rope":
        size = n * (case["heads"] + case["kv_heads"]) * case["dim"] * (2 if case["train"] else 1)
        return {"bytes": 2 * size * e + 4 * n * len(_parts(case)), "flops": 3 * size}
    c = float(case["c"])
    if case["kind"] == "norm":
        return {"bytes": (7 if case["residual"] else 4) * n * c * e + 4 * n + 8 * c, "flops": 14 * n * c}
    m = float(case["m"])
    weights = m * c + m * math.ceil(c / 128)                  # in 8 bits
    if case["kind"] == "serve":
        return {"bytes": 3 * n * c * e + 2 * n * m + weights + 4 * c, "flops": 2 * n * c * m}
    if case["kind"] == "q8":
        if case["train"]:
            return {"bytes": 2 * (n * c + n * m + m * c) * e, "flops": 6 * n * c * m}
        return {"bytes": (n * c + n * m) * e + weights, "flops": 2 * n * c * m}
    times = 2 if case["train"] else 1
    return {"bytes": times * (2 * n * c + 3 * m * c) * e, "flops": 6 * n * c * m * (3 if case["train"] else 1)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "norm": _exact_norm, "serve": _exact_serve, "q8": _exact_q8, "ffn": _exact_ffn}[case["kind"]](s)


def _exact_rope(s):
    """Every pair as a complex number, times e^(i angle); the gradient times the conjugate."""
    case = s["case"]

    def turned(x, sign):
        y, at = x.double().clone(), 0
        for a, part in enumerate(_parts(case)):
            if part:
                half = part // 2
                i = torch.arange(half, dtype=torch.float64, device="cuda")
                angle = sign * s["pos"][:, a].double()[:, None] * torch.exp(-math.log(10000.0) * 2 * i / part)
                block = y[:, :, at:at + part]
                z = torch.complex(block[..., :half], block[..., half:]) if case["split"] else torch.view_as_complex(
                    block.reshape(*block.shape[:2], half, 2).contiguous())
                z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
                y[:, :, at:at + part] = torch.cat([z.real, z.imag], 2) if case["split"] else torch.view_as_real(z).flatten(2)
            at += part
        return y

    out = {"y": turned(s["x"], 1)}
    if case["train"]:
        out["dx"] = turned(s["dy"], -1)
    return out


def _stored(s):
    """The sum with the residual, in 64 bits, as the storage type holds it."""
    h = s["x"].double()
    return h if s["res"] is None else (h + s["res"].double()).to(s["x"].dtype).double()


def _exact_norm(s):
    """The forward formula; the gradients come from differentiating it, some rows at a time."""
    h = _stored(s)
    gamma = s["gamma"].double().requires_grad_()
    ys, rs, dxs, dgamma = [], [], [], torch.zeros_like(gamma)
    rows = max(1, 20_000_000 // h.shape[1])
    for r in range(0, len(h), rows):
        x = h[r:r + rows].clone().requires_grad_()
        rstd = (x.square().mean(1) + 1e-5).rsqrt()
        y = x * rstd[:, None] * gamma
        loss = (y * s["dy"][r:r + rows].double()).sum()
        if s["dh"] is not None:
            loss = loss + (x * s["dh"][r:r + rows].double()).sum()
        dx, dg = torch.autograd.grad(loss, (x, gamma))
        ys.append(y.detach()), rs.append(rstd.detach()), dxs.append(dx)
        dgamma = dgamma + dg
    return {"h": h, "y": torch.cat(ys), "rstd": torch.cat(rs), "dx": torch.cat(dxs), "dgamma": dgamma.detach()}


def _grid(x):
    """x [n][c] (64 bits) as 8-bit elements with a power of two for each 128 of a row can hold it: 4 significant bits, exponents
    of elements down to -6, steps of 2^-9 below that."""
    n, c = x.shape
    out = torch.empty_like(x)
    for k in range(0, c, 128):
        b = x[:, k:k + 128]
        top = b.abs().amax(1, keepdim=True)
        unit = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, 448.0) / 448.0)).clamp(-127, 127))
        unit = torch.where(top > 448 * unit, 2 * unit, unit)  # where the logarithm's rounding hid a step
        unit = torch.where((top > 0) & (top <= 224 * unit) & (unit > 2.0 ** -127), unit / 2, unit)
        v = b / unit
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, k:k + 128] = torch.round(v / step) * step * unit
    return out


def _weights(s, c):
    return _from_q8(s["w"], c).double()                       # what is kept stands for just these values


def _exact_serve(s):
    h, c = _stored(s), s["case"]["c"]
    y = h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt() * s["gamma"].double()
    return {"h": h, "y": _grid(y) @ _weights(s, c).t()}


def _exact_q8(s):
    x, c = s["x"].double(), s["case"]["c"]
    if not s["case"]["train"]:
        return {"y": _grid(x) @ _weights(s, c).t()}
    w, dy = s["w"].double(), s["dy"].double()
    return {"y": _grid(x) @ _grid(w).t(), "dx": _grid(dy) @ _grid(w.t().contiguous()).t(),
            "dw": _grid(dy.t().contiguous()) @ _grid(x.t().contiguous()).t()}


def _exact_ffn(s):
    """The block as a function of rows and weights, some rows at a time; gradients by differentiation."""
    case = s["case"]
    m, train = case["m"], case["train"]
    w_in, w_out = (s[k].double().requires_grad_(train) for k in ("w_in", "w_out"))
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[case["act"]]
    ys, dxs, dw = [], [], [torch.zeros_like(w_in), torch.zeros_like(w_out)]
    rows = max(1, 50_000_000 // m)
    for r in range(0, case["n"], rows):
        x = s["x"][r:r + rows].double().requires_grad_(train)
        y = (act(x @ w_in[:m].t()) * (x @ w_in[m:].t())) @ w_out.t()
        ys.append(y.detach())
        if train:
            grads = torch.autograd.grad(y, (x, w_in, w_out), s["dy"][r:r + rows].double())
            dxs.append(grads[0])
            dw = [a + b for a, b in zip(dw, grads[1:])]
    out = {"y": torch.cat(ys)}
    if train:
        out.update(dx=torch.cat(dxs), dw_in=dw[0].detach(), dw_out=dw[1].detach())
    return out
