"""The operators of a transformer over the rows of a sparse tensor, as cases that can be timed and compared.

Kinds of pass
  norm     layer normalisation of [n][c] rows: forward, then the gradients of rows, weight and bias
  attend   attention over packed clouds (row ranges) with a sliding window and a few first rows that stay visible, on
           query / key / value views of one fused projection: forward, and in training the three gradients
  step     the same attention for one new token of each sequence, over a ring cache that the call also appends to
  distill  the loss against a teacher's top logits and its gradient

With `own` false a pass computes the operators in their plain form: products, sums, exponentials and indexing in 32 bits,
rounded once at the end.  With `own` true it makes the calls of paper_2012_13846_amd.binding.
"""
import math

import numpy as np
import torch

own = False


# ---- the cases -------------------------------------------------------------------------------------------------
def _norm(n, c, dtype):
    return {"kind": "norm", "n": n, "c": c, "dtype": dtype}


def _attend(clouds, total, heads, kv_heads, dim, left, right, sinks, dtype, train, queries=0):
    """total keys over all clouds; queries: the last rows of each cloud that ask (0: all of them)."""
    return {"kind": "attend", "clouds": clouds, "total": total, "heads": heads, "kv_heads": kv_heads, "dim": dim, "left": left,
            "right": right, "sinks": sinks, "dtype": dtype, "train": train, "queries": queries}


def _step(batch, heads, kv_heads, dim, left, sinks, cap, most, dtype):
    return {"kind": "step", "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "left": left, "sinks": sinks, "cap": cap,
            "most": most, "dtype": dtype}


def _distill(n, m, k, temperature, weighted, dtype):
    return {"kind": "distill", "n": n, "m": m, "k": k, "temperature": temperature, "weighted": weighted, "dtype": dtype}


def listed():
    return [
        # one object at the coarsest grid: launches and latency
        {"name": "norm_one_shape_c128_bf16", **_norm(1428, 128, "bf16")},
        # a micro-batch of four fine clouds at the classifier's last width
        {"name": "norm_batch4_c256_bf16", **_norm(373601, 256, "bf16")},
        # a width that is no whole number of 16-byte pieces
        {"name": "norm_odd_c77_f32", **_norm(70001, 77, "f32")},
        # wide rows of a token model
        {"name": "norm_wide_c4096_bf16", **_norm(16384, 4096, "bf16")},
        # eight small clouds of a batch, full precision: launches and latency
        {"name": "attend_small_d16_f32", **_attend(8, 1601, 4, 4, 16, 64, 64, 1, "f32", True)},
        # training on the rows of four fine clouds, windows to both sides
        {"name": "attend_batch4_d32_bf16", **_attend(4, 373601, 8, 8, 32, 256, 256, 4, "bf16", True)},
        # training a causal token model with shared key/value heads on two documents of unlike length
        {"name": "attend_causal_h32kv8_d128_bf16", **_attend(2, 16384, 32, 8, 128, 1023, 0, 4, "bf16", True)},
        # reading the next part of long prompts: 2048 queries of each against what came before, forward only
        {"name": "attend_prompt_d64_bf16", **_attend(3, 100003, 16, 4, 64, 4095, 0, 16, "bf16", False, 2048)},
        # one user's next token far into a session: latency
        {"name": "step_b1_h32kv8_d128_bf16", **_step(1, 32, 8, 128, 4095, 4, 4100, 200000, "bf16")},
        # a serving batch, sequences of every length
        {"name": "step_b96_h32kv8_d128_bf16", **_step(96, 32, 8, 128, 4095, 4, 4100, 30000, "bf16")},
        # per-voxel distillation of a segmentation net: 40 categories, the teacher's five best
        {"name": "distill_voxels_m40_f32", **_distill(160000, 40, 5, 2.0, True, "f32")},
        # a large vocabulary
        {"name": "distill_m131072_bf16", **_distill(4096, 131072, 64, 1.0, False, "bf16")},
    ]


def draw(rng):
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "norm", "attend", "attend", "attend", "step", "distill", "distill"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "norm":
        c = rng.choice([span(16, 8192), 8 * span(2, 1024), rng.choice([32, 64, 128, 256, 512, 1024, 2048])])
        return _norm(span(1, min(400000, 40_000_000 // c)), c, dtype)
    if kind == "attend":
        dim = rng.choice([16, 32, 48, 64, 64, 80, 96, 128, 128, rng.randint(1, 128)])
        kv = rng.choice([1, 2, 3, 4, 8])
        heads = kv * rng.choice([1, 1, 2, 4, 5])
        left = span(1, 4096)
        right = rng.choice([0, 0, left, span(1, 512)])
        sinks = rng.choice([0, 1, 4, 17, 64])
        # rows x what they see x heads x dim stays below a quarter of the listed training cases' (an eighth of it in fp32)
        most = 60_000_000_000 // (left + right + 1 + sinks) // (heads * (dim + 16)) // (16 if dtype == "f32" else 2)
        total = span(1 if rng.random() < 0.2 else 64, max(65, min(100000, most)))
        clouds = min(span(1, 64), total)
        train = rng.random() < 0.7
        return _attend(clouds, total, heads, kv, dim, left, right, sinks, dtype, train, 0 if train else rng.choice([0, 1, span(1, 1024)]))
    if kind == "step":
        kv = rng.choice([1, 2, 4, 8])
        dim = rng.choice([32, 64, 80, 128, 128, rng.randint(1, 128)])
        sinks = rng.choice([0, 1, 4, 17])
        left = span(1, 4096)
        most = span(16, 30000)
        cap = rng.choice([sinks + left + 1, sinks + left + span(1, 512), min(8192, max(most, sinks + left) + 1)])
        room = 400_000_000 // (cap * kv * dim)
        return _step(span(1, max(1, min(128, room))), kv * rng.choice([1, 2, 4, 7, 8]), kv, dim, left, sinks, cap, most, dtype)
    m = rng.choice([span(8, 200000), 8 * span(4, 16384), rng.choice([40, 1000, 32000, 65536])])
    k = min(m, rng.choice([1, 5, 10, 32, 64, 100]))
    return _distill(span(1, max(1, min(200000, 250_000_000 // m))), m, k, rng.choice([1.0, 2.0, 4.0]), rng.random() < 0.5, dtype)


# ---- what a program holds before the call ----------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """Keys and queries of each cloud: unlike lengths that add up to the total (by the case alone, not by the seed)."""
    clouds, total = case["clouds"], case["total"]
    rng = np.random.default_rng(clouds * 1_000_003 + total)
    cuts = np.sort(rng.integers(0, total + 1, clouds - 1)) if clouds > 64 else None
    if cuts is None:
        share = rng.uniform(0.6, 1.4, clouds)
        cuts = np.floor(np.cumsum(share)[:-1] / share.sum() * total).astype(np.int64)
    b = np.diff(np.concatenate([[0], cuts, [total]]))
    a = b if not case["queries"] else np.minimum(b, case["queries"])
    return [int(v) for v in a], [int(v) for v in b]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    s = {"case": case}
    if case["kind"] == "norm":
        n, c = case["n"], case["c"]
        s["x"] = (1.5 * normal(n, c) + 0.5 * normal(n, 1)).to(dt)     # rows have means of their own
        s["dy"] = normal(n, c).to(dt)
        s["gamma"], s["beta"] = 1 + 0.2 * normal(c), 0.2 * normal(c)
    elif case["kind"] == "attend":
        a, b = _lengths(case)
        h, kv, d = case["heads"], case["kv_heads"], case["dim"]
        s["q_lens"], s["k_lens"] = a, b
        for name, lens in (("q_starts", a), ("k_starts", b)):
            s[name] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
        if a == b:                                                    # one projection gives all three
            w = normal(sum(b), h + 2 * kv, d).to(dt)
            s["q"], s["k"], s["v"] = w[:, :h], w[:, h:h + kv], w[:, h + kv:]
        else:                                                         # keys and values come from a cache
            s["q"], w = normal(sum(a), h, d).to(dt), normal(sum(b), 2 * kv, d).to(dt)
            s["k"], s["v"] = w[:, :kv], w[:, kv:]
        if case["train"]:
            s["do"] = normal(sum(a), h, d).to(dt)
    elif case["kind"] == "step":
        n, h, kv, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
        s["q"], s["k_new"], s["v_new"] = normal(n, h, d).to(dt), normal(n, kv, d).to(dt), normal(n, kv, d).to(dt)
        s["k_cache"] = torch.empty((n, case["cap"], kv, d), dtype=dt, device="cuda").normal_(generator=g)
        s["v_cache"] = torch.empty((n, case["cap"], kv, d), dtype=dt, device="cuda").normal_(generator=g)
        most = case["most"]                                           # the first sequence is the longest; some have just begun
        lens = (most * torch.rand(n, device="cuda", generator=g) ** 1.5).to(torch.int32)
        lens[0] = most
        if n > 4:
            lens[1], lens[2] = 0, -1                                  # one before its first token, one slot without a sequence
        s["lens"] = lens
    else:
        n, m, k = case["n"], case["m"], case["k"]
        index = torch.arange(k, device="cuda") * (m // k) + torch.randint(0, m // k, (n, k), device="cuda", generator=g)
        t = (4 + 2 * normal(n, k)).sort(dim=1, descending=True).values
        z = torch.empty((n, m), dtype=dt, device="cuda").normal_(0, 2, generator=g)
        z.scatter_(1, index, (t + normal(n, k)).to(dt))               # a student that has learnt some of it
        held = torch.randint(0, 16 * k, (n, 1), device="cuda", generator=g)   # one row in 16 has fewer entries or none
        s["index"] = torch.where(torch.arange(k, device="cuda") < held, index, -1).to(torch.int32)
        s["t"], s["z"] = t, z
        s["weight"] = torch.rand(n, device="cuda", generator=g) / n if case["weighted"] else None
    return s


# ---- one pass --------------------------------------------------------------------------------------------------
def _run_own(s):
    from paper_2012_13846_amd import binding as sp
    case = s["case"]
    if case["kind"] == "norm":
        y, mean, rstd = sp.sp_layer_norm_fwd(s["x"], s["gamma"], s["beta"], 1e-5)
        dx, dgamma, dbeta = sp.sp_layer_norm_bwd(s["x"], s["dy"], s["gamma"], mean, rstd)
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if case["kind"] == "attend":
        shape = dict(left=case["left"], right=case["right"], sinks=case["sinks"])
        o, lse = sp.sp_window_attn_fwd(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], **shape)
        out = {"o": o, "lse": lse}
        if case["train"]:
            out["dq"], out["dk"], out["dv"] = sp.sp_window_attn_bwd(s["q"], s["k"], s["v"], o, s["do"], lse, s["q_starts"], s["k_starts"],
                                                                    **shape)
        return out
    if case["kind"] == "step":
        o = sp.sp_window_attn_step(s["q"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["lens"], left=case["left"],
                                   sinks=case["sinks"])
        return {"o": o, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    loss, dz = sp.sp_distill(s["z"], s["t"], s["index"], temperature=case["temperature"], weight=s["weight"])
    return {"loss": loss, "dz": dz}


def run(s):
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "attend": _plain_attend, "step": _plain_step, "distill": _plain_distill}[s["case"]["kind"]](s)


def _plain_norm(s):
    dt, c = s["x"].dtype, s["x"].shape[1]
    x, dy = s["x"].float(), s["dy"].float()
    mean = x.sum(1, keepdim=True) / c
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).sum(1, keepdim=True) / c + 1e-5)
    xh = d * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - g.sum(1, keepdim=True) / c - xh * ((g * xh).sum(1, keepdim=True) / c))
    return {"y": (xh * s["gamma"] + s["beta"]).to(dt), "mean": mean[:, 0], "rstd": rstd[:, 0], "dx": dx.to(dt), "dgamma": (dy * xh).sum(0),
            "dbeta": dy.sum(0)}


def _plain_attend(s):
    """Blocks of queries against the keys that any of them sees: the first ones and one stretch."""
    case, dt = s["case"], s["q"].dtype
    h, kv, d, left, right, sinks = (case[n] for n in ("heads", "kv_heads", "dim", "left", "right", "sinks"))
    per, scale = h // kv, 1 / math.sqrt(d)
    n_q, n_k = s["q"].shape[0], s["k"].shape[0]
    train = case["train"]
    o = torch.zeros((n_q, h, d), device="cuda")
    lse = torch.full((n_q, h), -math.inf, device="cuda")
    if train:
        dq = torch.zeros((n_q, h, d), device="cuda")
        dk, dv = torch.zeros((n_k, kv, d), device="cuda"), torch.zeros((n_k, kv, d), device="cuda")
    block = max(256, min(1024, left + right))
    q0 = k0 = 0
    for a, b in zip(s["q_lens"], s["k_lens"]):
        for i0 in range(0, a, block):
            i1 = min(a, i0 + block)
            p = torch.arange(i0 + b - a, i1 + b - a, device="cuda")[:, None]
            lo, hi = max(0, i0 + b - a - left), min(b, i1 + b - a + right)
            first = min(sinks, lo, hi)
            j = torch.cat([torch.arange(first, device="cuda"), torch.arange(lo, max(lo, hi), device="cuda")])
            seen = (j <= p + right) & ((j >= p - left) | (j < sinks))                              # [queries][keys]

            def heads_first(t, n):                                                                # [rows][n][d] -> [n][rows][d]
                return t.float().transpose(0, 1).contiguous()

            def grouped(t):                                                                       # -> [kv][per * queries][d]
                return heads_first(t[q0 + i0:q0 + i1], h).view(kv, per * (i1 - i0), d)

            q, k, v = grouped(s["q"]), heads_first(s["k"][k0 + j], kv), heads_first(s["v"][k0 + j], kv)
            sc = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
            sc = sc.masked_fill_(~seen.repeat(per, 1), -math.inf)
            top = sc.amax(2, keepdim=True)
            e = torch.exp(sc - top)
            total = e.sum(2, keepdim=True)
            e = e / total
            out = torch.matmul(e, v)

            def rows(t):                                                                          # [kv][per * queries][..] -> rows first
                return t.view(h, i1 - i0, -1).transpose(0, 1)

            o[q0 + i0:q0 + i1] = rows(out)
            lse[q0 + i0:q0 + i1] = rows(top + torch.log(total))[:, :, 0]
            if train:
                do = grouped(s["do"])
                ds = e * (torch.matmul(do, v.transpose(1, 2).contiguous()) - (do * out).sum(2, keepdim=True)) * scale
                dq[q0 + i0:q0 + i1] = rows(torch.matmul(ds, k))
                dk[k0 + j] += torch.matmul(ds.transpose(1, 2).contiguous(), q).transpose(0, 1)
                dv[k0 + j] += torch.matmul(e.transpose(1, 2).contiguous(), do).transpose(0, 1)
        q0, k0 = q0 + a, k0 + b
    r = {"o": o.to(dt), "lse": lse}
    if train:
        r.update(dq=dq.to(dt), dk=dk.to(dt), dv=dv.to(dt))
    return r


def _plain_step(s):
    case, dt = s["case"], s["q"].dtype
    h, kv, d, left, sinks, cap = (case[n] for n in ("heads", "kv_heads", "dim", "left", "sinks", "cap"))
    n, ring = case["batch"], case["cap"] - case["sinks"]
    p = s["lens"].long()
    live = p >= 0
    at = torch.where(p < sinks, p, sinks + (p - sinks) % ring).clamp_(min=0)
    row = torch.arange(n, device="cuda")
    for cache, new in ((s["k_cache"], s["k_new"]), (s["v_cache"], s["v_new"])):
        cache[row, at] = torch.where(live[:, None, None], new, cache[row, at])
    slot = torch.arange(cap, device="cuda")
    # the last position that lies in this slot of the ring
    pos = torch.where(slot < sinks, slot, p[:, None] - (p[:, None] - slot) % ring)
    seen = live[:, None] & (pos <= p[:, None]) & (pos >= 0) & ((pos >= p[:, None] - left) | (pos < sinks)) & ((slot < sinks) | (pos >= sinks))
    q = s["q"].float().view(n, kv, h // kv, d) / math.sqrt(d)
    k = s["k_cache"].float().permute(0, 2, 3, 1).contiguous()
    sc = torch.matmul(q, k).masked_fill_(~seen[:, None, None], -math.inf)
    top = sc.amax(3, keepdim=True).clamp_(min=-3e38)
    e = torch.exp(sc - top)
    out = torch.matmul(e / e.sum(3, keepdim=True).clamp_(min=1e-30), s["v_cache"].float().transpose(1, 2).contiguous())
    return {"o": out.view(n, h, d).to(dt), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_distill(s):
    case, temp = s["case"], s["case"]["temperature"]
    n = case["n"]
    there = (s["index"] >= 0) & (s["index"] < case["m"])
    some = there.any(1, keepdim=True)
    index = torch.where(there, s["index"], 0).long()
    t = torch.where(there, s["t"] / temp, -math.inf)
    t = t - torch.where(some, t.amax(1, keepdim=True), 0.0)
    e = torch.exp(t)
    total = e.sum(1, keepdim=True).clamp_(min=1e-30)
    a = e / total
    z = s["z"].float() / temp
    top = z.amax(1, keepdim=True)
    ez = torch.exp(z - top)
    sum_z = ez.sum(1, keepdim=True)
    terms = torch.where(a > 0, a * (t - torch.log(total) - z.gather(1, index) + top + torch.log(sum_z)), 0.0)
    w = s["weight"] if s["weight"] is not None else torch.full((n,), 1 / n, device="cuda")
    loss = (w.double() * terms.sum(1).double()).sum() * temp * temp
    dz = (ez / sum_z * some).scatter_add_(1, index, -a) * (w * temp)[:, None]
    return {"loss": loss.float().view(1), "dz": dz.to(s["z"].dtype)}


# ---- what a pass cannot do without -----------------------------------------------------------------------------
def _pairs(a, b, case):
    """Query-key pairs that are seen."""
    p = np.arange(a, dtype=np.int64) + (b - a)
    hi = np.clip(p + case["right"] + 1, 0, b)
    lo = np.minimum(np.clip(p - case["left"], 0, b), hi)
    return int((hi - lo + np.minimum(np.minimum(case["sinks"], lo), hi)).sum())


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "norm":
        n, c = case["n"], case["c"]
        return {"bytes": 4.0 * n * c * e + 8.0 * n + 20.0 * c, "flops": 22.0 * n * c}
    if case["kind"] == "attend":
        a, b = _lengths(case)
        h, kv, d = case["heads"], case["kv_heads"], case["dim"]
        pairs = sum(_pairs(x, y, case) for x, y in zip(a, b))
        q, k = float(sum(a)) * h * d * e, float(sum(b)) * kv * d * e
        if not case["queries"]:
            byts = 2 * q + 2 * k
        else:                                             # keys far behind every query are not touched
            reach = sum(min(y, x + case["left"] + case["sinks"]) for x, y in zip(a, b))
            byts = 2 * q + 2.0 * reach * kv * d * e
        byts += 4.0 * sum(a) * h
        flops = 4.0 * pairs * h * d
        if case["train"]:
            byts, flops = byts + 2 * q + 2 * k, 3.5 * flops
        return {"bytes": byts, "flops": flops}
    if case["kind"] == "step":
        n, h, kv, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
        u = np.linspace(0, 1, 1001)
        lens = case["most"] * u ** 1.5 if n > 1 else np.array([case["most"]])
        seen = np.minimum(lens + 1, min(case["left"] + 1, case["cap"] - case["sinks"]) + case["sinks"]).mean() * n
        return {"bytes": 2.0 * seen * kv * d * e + 2.0 * n * (h + kv) * d * e, "flops": 4.0 * seen * h * d}
    n, m, k = case["n"], case["m"], case["k"]
    return {"bytes": 2.0 * n * m * e + 8.0 * n * k, "flops": 8.0 * n * m}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "attend": _exact_attend, "step": _exact_step, "distill": _exact_distill}[case["kind"]](s)


def _exact_norm(s):
    """The forward formula; the gradients come from differentiating it, some rows at a time."""
    gamma, beta = s["gamma"].double().requires_grad_(), s["beta"].double().requires_grad_()
    n, c = s["x"].shape
    y, dx, stat = torch.empty((n, c), dtype=torch.float64, device="cuda"), torch.empty((n, c), dtype=torch.float64, device="cuda"), []
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
    rows = max(1, 20_000_000 // c)
    for r in range(0, n, rows):
        x = s["x"][r:r + rows].double().requires_grad_()
        mean = x.mean(1)
        rstd = ((x - mean[:, None]).square().mean(1) + 1e-5) ** -0.5
        out = (x - mean[:, None]) * rstd[:, None] * gamma + beta
        grads = torch.autograd.grad(out, (x, gamma, beta), s["dy"][r:r + rows].double())
        y[r:r + rows], dx[r:r + rows] = out.detach(), grads[0]
        dgamma, dbeta = dgamma + grads[1], dbeta + grads[2]
        stat.append((mean.detach(), rstd.detach()))
    return {"y": y, "mean": torch.cat([m for m, _ in stat]), "rstd": torch.cat([r for _, r in stat]), "dx": dx, "dgamma": dgamma.detach(),
            "dbeta": dbeta.detach()}


def _exact_attend(s):
    """Softmax over the visible keys of every query, one cloud, head and block of queries at a time; gradients by differentiation."""
    case = s["case"]
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    a, b = s["q_lens"], s["k_lens"]
    pairs = sum(_pairs(x, y, case) for x, y in zip(a, b))
    block = 512
    calls = h * sum((x + block - 1) // block for x in a)
    if pairs * h * (d + 60) * (4 if case["train"] else 1) > 1e13 or calls * (2e-3 if case["train"] else 1e-3) > 16:
        return None
    n_q, n_k = s["q"].shape[0], s["k"].shape[0]

    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.float64, device="cuda")

    o, lse, dq, dk, dv = zeros(n_q, h, d), zeros(n_q, h), zeros(n_q, h, d), zeros(n_k, kv, d), zeros(n_k, kv, d)
    q0 = k0 = 0
    for x, y in zip(a, b):
        for i in range(0, x, block):
            n = min(block, x - i)
            stand = i + y - x                                       # where the block's first query stands among the keys
            end = max(0, min(y, stand + n + case["right"]))
            begin = min(end, max(0, stand - case["left"]))
            keys = torch.tensor(list(range(min(begin, case["sinks"]))) + list(range(begin, end)), dtype=torch.int64, device="cuda")
            away = keys[None, :] - (stand + torch.arange(n, device="cuda"))[:, None]
            hidden = (away > case["right"]) | ((away < -case["left"]) & (keys[None, :] >= case["sinks"]))
            for c in range(h):
                at = slice(q0 + i, q0 + i + n)
                if not len(keys):
                    lse[at, c] = -math.inf
                    continue
                q, k, v = (t.double().requires_grad_(case["train"]) for t in
                           (s["q"][at, c], s["k"][k0 + keys, c // (h // kv)], s["v"][k0 + keys, c // (h // kv)]))
                score = (q @ k.t()) * d ** -0.5
                none = hidden.all(1, keepdim=True)
                score = torch.where(hidden, -math.inf, score)
                prob = torch.softmax(torch.where(none, 0.0, score), 1) * ~none
                out = prob @ v
                o[at, c], lse[at, c] = out.detach(), torch.logsumexp(score.detach(), 1)
                if case["train"]:
                    gq, gk, gv = torch.autograd.grad(out, (q, k, v), s["do"][at, c].double())
                    dq[at, c] = gq
                    dk[k0 + keys, c // (h // kv)] += gk
                    dv[k0 + keys, c // (h // kv)] += gv
        q0, k0 = q0 + x, k0 + y
    r = {"o": o, "lse": lse}
    if case["train"]:
        r.update(dq=dq, dk=dk, dv=dv)
    return r


def _exact_step(s):
    """One sequence at a time: which positions are seen, where each lies, and the softmax over them."""
    case = s["case"]
    h, kv, d, sinks, ring = case["heads"], case["kv_heads"], case["dim"], case["sinks"], case["cap"] - case["sinks"]
    out = torch.zeros((case["batch"], h, d), dtype=torch.float64, device="cuda")
    for i, p in enumerate(s["lens"].tolist()):
        if p < 0:
            continue
        where = lambda j: j if j < sinks else sinks + (j - sinks) % ring  # noqa: E731
        s["k_cache"][i, where(p)], s["v_cache"][i, where(p)] = s["k_new"][i], s["v_new"][i]
        low = max(p - case["left"], p + 1 - ring)
        slots = torch.tensor([where(j) for j in range(p + 1) if j < sinks or j >= low] if p < 20000 else
                             [where(j) for j in range(min(sinks, p + 1))] + [where(j) for j in range(max(low, sinks), p + 1)], device="cuda")
        k, v = s["k_cache"][i, slots].double(), s["v_cache"][i, slots].double()
        for c in range(h):
            score = k[:, c // (h // kv)] @ s["q"][i, c].double() / d ** 0.5
            out[i, c] = torch.softmax(score, 0) @ v[:, c // (h // kv)]
    return {"o": out, "k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}


def _exact_distill(s):
    """The divergence of every row's two distributions; the gradient by differentiation, some rows at a time."""
    case, temp = s["case"], s["case"]["temperature"]
    n, m = s["z"].shape
    dz, loss = torch.empty((n, m), dtype=torch.float64, device="cuda"), 0.0
    rows = max(1, 30_000_000 // m)
    for r in range(0, n, rows):
        z = s["z"][r:r + rows].double().requires_grad_()
        index = s["index"][r:r + rows].long()
        real = (index >= 0) & (index < m)
        teacher = torch.softmax(torch.where(real, s["t"][r:r + rows].double() / temp, -1e300), 1) * real
        student = torch.log_softmax(z / temp, 1).gather(1, torch.where(real, index, 0))
        w = s["weight"][r:r + rows].double() if s["weight"] is not None else torch.full((len(z),), 1 / n, dtype=torch.float64, device="cuda")
        part = (w[:, None] * (torch.special.xlogy(teacher, teacher) - teacher * student)).sum() * temp ** 2
        dz[r:r + rows] = torch.autograd.grad(part, z)[0]
        loss += float(part.detach())
    return {"loss": torch.tensor([loss], dtype=torch.float64, device="cuda"), "dz": dz}
