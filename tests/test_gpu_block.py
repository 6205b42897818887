"""Rotary positions, root-mean-square norm, rows and products in 8 bits and the gated feed-forward block on the GPU against
oracle/block.py (float64).

Tolerances are bounds of the error, element by element, from half a step of the storage type (u) and of fp32 (U32 = 2^-24)
relative to each rounded value, as derived beside each comparison.
"""
import math

import numpy as np
import pytest
import torch

from oracle import block

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U32 = torch.finfo(F32).eps / 2
TYPES = pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])


@pytest.fixture(scope="module")
def sp():
    from paper_2012_13846_amd import binding
    binding.lib()
    return binding


def half_step(dt):
    return torch.finfo(dt).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def rows(rng, dt, *shape, scale=1.0):
    """Values of the storage type, on the GPU (read back exactly by host)."""
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dt).cuda()


def within(got, want, bound, what):
    within_values(host(got), np.asarray(want), bound, what)


def within_values(got, want, bound, what):
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), f"{what}: finite in other places"
    over = np.abs(got[fine] - want[fine]) - np.broadcast_to(bound, want.shape)[fine]
    assert over.size == 0 or over.max() <= 0, f"{what}: {over.max():.3e} over its bound"


# ---- rotary positions ------------------------------------------------------------------------------------------
# rows, heads, dim, parts, positions up to
ROPE = {
    "one": (1, 1, 2, (2,), 10),
    "token": (3, 5, 64, (64,), 200000),
    "xyz": (77, 4, 32, (12, 10, 10), 500),
    "xyz_even": (130, 3, 96, (32, 32, 32), 40),
    "video": (65, 2, 128, (16, 48, 32, 32), 1000),
    "some_stay": (33, 3, 80, (16, 32), 3000),
    "none_turns": (9, 2, 16, (0, 0), 30),
    "an_axis_of_none": (31, 2, 24, (8, 0, 8), 30),
    "odd": (41, 3, 33, (10, 22), 1 << 20),
    "wide": (19, 2, 256, (256,), 1 << 30),
    "far": (50, 1, 48, (48,), (1 << 31) - 1),
    "many": (5000, 8, 16, (4, 6, 6), 300),
    "many_heads": (7, 130, 6, (6,), 300),
}


def rope_bound(x, y, pos, parts, split, scale, u):
    """cosine and sine: the angle in turns, rounded to fp32 (half a step of a value up to 1/2, times 2 pi), and two steps of sincospi: 6 U32; the
    frequency and the product in fp64 here and there: 6 * 2^-53 of the angle.  Two products and a sum: 3 U32.  Then the storage type."""
    size, at = np.zeros_like(x), 0
    for part in parts:
        for i in range(part // 2):
            j, k = (at + i, at + i + part // 2) if split else (at + 2 * i, at + 2 * i + 1)
            size[:, :, j] = size[:, :, k] = np.abs(x[:, :, j]) + np.abs(x[:, :, k])
        at += part
    far = np.abs(pos.astype(np.float64)).max(initial=0) * abs(scale)
    return size * (9 * U32 + 16 * 2.0 ** -53 * far) + np.where(size > 0, (u + U32) * np.abs(y), 0)


@TYPES
@pytest.mark.parametrize("split", [False, True], ids=["neighbours", "halves"])
@pytest.mark.parametrize("case", ROPE)
def test_rope(sp, case, split, dt):
    n, heads, dim, parts, far = ROPE[case]
    rng = np.random.default_rng(n + dim)
    w = rows(rng, dt, n, heads + 2, dim)
    x = w[:, 1:heads + 1] if heads > 1 else w[:, :1]        # heads of a fused projection
    pos = torch.from_numpy(rng.integers(-far, far, (n, len(parts) + 1)).astype(np.int32)).cuda()[:, 1:]
    p, u = pos.cpu().numpy(), (half_step(dt) if dt == BF16 else 0)
    y = sp.sp_rope_fwd(x, pos, parts, split=split, base=500.0, scale=0.25)
    Y = block.rope(host(x), p, parts, 500.0, split, 0.25)
    within(y, Y, rope_bound(host(x), Y, p, parts, split, 0.25, u), "y")
    dx = sp.sp_rope_bwd(x, pos, parts, split=split, base=500.0, scale=0.25)
    DX = block.rope(host(x), p, parts, 500.0, split, 0.25, back=True)
    within(dx, DX, rope_bound(host(x), DX, p, parts, split, 0.25, u), "dx")
    # in place, in the projection: the same bits, and nothing else is written
    before = w.clone()
    got = sp.sp_rope_fwd(x, pos, parts, split=split, base=500.0, scale=0.25, out=x)
    assert got.data_ptr() == x.data_ptr() and torch.equal(x, y)
    a = 1 if heads > 1 else 0
    assert torch.equal(w[:, :a], before[:, :a]) and torch.equal(w[:, a + heads:], before[:, a + heads:])


def test_rope_of_a_sparse_tensors_coordinates(sp):
    from paper_2012_13846_amd import spgen
    coords = sp.sp_coords_build(torch.from_numpy(spgen.coords_config(1, 0.02)).cuda(), 1)
    x = torch.randn((coords.n, 2, 32), device="cuda")
    y = sp.sp_rope_fwd(x, coords.coords()[:, 1:], (12, 10, 10))
    p = coords.coords()[:, 1:].cpu().numpy()
    Y = block.rope(host(x), p, (12, 10, 10))
    within(y, Y, rope_bound(host(x), Y, p, (12, 10, 10), False, 1.0, 0), "y")


def test_rope_edges(sp):
    pos = torch.zeros((4, 1), dtype=torch.int32, device="cuda")
    x = torch.randn((4, 2, 8), device="cuda")
    x[1, 0, 3], x[2, 1, 7] = float("inf"), float("nan")
    y = sp.sp_rope_fwd(x, pos, (6,))
    fine = torch.ones_like(x, dtype=torch.bool)
    fine[1, 0, 2:4] = False                                  # its pair: infinity times a sine of zero is NaN
    fine[2, 1, 7] = False
    assert torch.equal(y[fine], x[fine]) and torch.isnan(y[2, 1, 7])
    assert sp.sp_rope_fwd(x[:0], pos[:0], (6,)).shape == (0, 2, 8)
    flat = torch.randn(4 * 16 + 1, device="cuda")            # off a 16-byte border
    far = torch.arange(4, dtype=torch.int32, device="cuda")[:, None] * 77
    a = sp.sp_rope_fwd(flat[1:].view(4, 2, 8), far, (8,), split=True)
    assert torch.equal(a, sp.sp_rope_fwd(flat[1:].clone().view(4, 2, 8), far, (8,), split=True))
    for bad in (dict(pos=pos.long()), dict(pos=pos[:3]), dict(pos=pos.cpu()), dict(parts=(6, 2)), dict(parts=(10,)), dict(parts=()),
                dict(x=x.transpose(1, 2)), dict(x=x.cpu()), dict(x=x.double()), dict(out=x[:, :1])):
        args = dict(x=x, pos=pos, parts=(6,))
        args.update(bad)
        with pytest.raises(ValueError):
            sp.sp_rope_fwd(**args)
    with pytest.raises(sp.SpError):
        sp.sp_rope_fwd(x, pos, (5,))


# ---- root-mean-square norm -------------------------------------------------------------------------------------
NORM = [(1, 1), (1, 16), (3, 5), (1428, 128), (515, 77), (130, 64), (33, 1000), (257, 1024), (65, 2048), (19, 4096), (5, 8192), (4, 8191), (40, 72),
        (3, 16384), (2, 16392), (2, 40001), (7, 513), (40, 24), (9, 2056), (6, 4100), (20001, 8), (11, 130), (3, 65536)]


def sum_error(c):
    """Relative error of a sum of c squares: up to 16 (or, of rows that no registers hold, c / 1024) one after another, ten steps of lanes and
    wavefronts and four more, and the square's own rounding."""
    return (max(16, c / 1024 + 8) + 15) * U32


@TYPES
@pytest.mark.parametrize("n,c", NORM)
def test_rms_norm(sp, n, c, dt):
    rng = np.random.default_rng(n * 7 + c)
    x, res, dy, dh = (rows(rng, dt, n, c) for _ in range(4))
    gamma = 1 + rows(rng, F32, c, scale=0.2)
    eps, u, G = 1e-5, half_step(dt), host(gamma)
    for residual in (res, None):
        h, y, rstd = sp.sp_rms_norm_fwd(x, gamma, residual, eps)
        stored = x if residual is None else (x.float() + res.float()).to(dt)
        assert torch.equal(h, stored)
        H = host(h)
        Y, R = block.rms_fwd(H, G, eps)
        rel = sum_error(c) / 2 + 4 * U32                    # the root halves it; mean, root and quotient
        within(rstd, R, rel * R, "rstd")
        within(y, Y, (rel + 3 * U32 + u) * np.abs(Y), "y")
        # backward from the GPU's own rstd: the formula's inputs are exact then
        DH = None if residual is None else host(dh)
        dx, dgamma = sp.sp_rms_norm_bwd(h, dy, gamma, rstd, None if residual is None else dh)
        DX, DG = block.rms_bwd(H, host(dy), G, host(rstd), DH)
        R, hat, g = host(rstd)[:, None], np.abs(H * host(rstd)[:, None]), np.abs(host(dy) * G)
        mean = (g * hat).mean(1)[:, None]
        size = R * (g + hat * mean)
        within(dx, DX, (sum_error(c) + 6 * U32) * size + (0 if DH is None else U32 * np.abs(DH)) + (u + U32) * np.abs(DX), "dx")
        # the rows' sums: up to 1100 rows one after another in a lane or a column, the workgroups' sums in fp64
        run = (12 + min(n, 1100)) * U32
        within(dgamma, DG, run * np.abs(host(dy) * hat).sum(0) + U32 * np.abs(DG), "dgamma")


@TYPES
@pytest.mark.parametrize("n,c", NORM)
def test_rms_norm_in_8_bits(sp, n, c, dt):
    rng = np.random.default_rng(n * 5 + c)
    x, res = rows(rng, dt, n, c), rows(rng, dt, n, c)
    gamma = 1 + rows(rng, F32, c, scale=0.2)
    h, (codes, scales) = sp.sp_rms_norm_q8(x, gamma, res, 1e-5)
    assert torch.equal(h, (x.float() + res.float()).to(dt))
    wide = -(-c // 128) * 128
    q, s = codes.view(torch.uint8).cpu().numpy(), scales.view(torch.uint8).cpu().numpy()
    assert q.shape == (n, wide) and s.shape == (n, -(-wide // 512) * 4)
    assert not q[:, c:].any() and (s[:, wide // 128:] == 127).all()
    Y, _ = block.rms_fwd(host(h), host(gamma), 1e-5)
    err = (sum_error(c) / 2 + 7 * U32) * np.abs(Y)          # before the codes' rounding, as above
    V = block.q8_values(q, s)[:, :c]
    unit = np.repeat(2.0 ** (s[:, :wide // 128].astype(float) - 127), 128, axis=1)[:, :c]
    # half a step of a code: 2^-4 of the value, or of the smallest step, 2^-9 of the scale
    assert (np.abs(V - Y) <= err + np.maximum((np.abs(Y) + err) / 16, unit * 2.0 ** -10)).all()
    for b in range(wide // 128):                             # the least scale that holds the block
        top = np.abs(Y[:, 128 * b:128 * b + 128]).max(1)
        one = 2.0 ** (s[:, b].astype(float) - 127)
        slack = 1 + sum_error(c) / 2 + 7 * U32
        assert ((top <= 448 * one * slack) & (top * slack > 224 * one)).all()
    h2, (codes2, scales2) = sp.sp_rms_norm_q8(h, gamma)      # of the sum itself, without a residual
    assert h2 is h and torch.equal(codes2.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(scales2.view(torch.uint8), scales.view(torch.uint8))


def test_rms_norm_edges(sp):
    gamma = torch.ones(48, device="cuda")
    empty = torch.empty((0, 48), device="cuda")
    h, y, rstd = sp.sp_rms_norm_fwd(empty, gamma, empty)
    dx, dgamma = sp.sp_rms_norm_bwd(h, empty, gamma, rstd)
    assert y.shape == (0, 48) and dx.shape == (0, 48) and not dgamma.any()
    assert sp.sp_rms_norm_q8(empty, gamma)[1][0].shape == (0, 128)
    x = torch.randn((7, 48), device="cuda")
    x[2, 5], x[4, 0] = float("nan"), float("inf")
    x[5] = 0
    x[6] = 3e30                                              # squares beyond fp32
    h, y, rstd = sp.sp_rms_norm_fwd(x, gamma)
    assert h is x and torch.isnan(y[2]).all() and torch.isnan(y[4, 0]) and not y[4, 1:].any() and not y[5].any()
    assert torch.isfinite(y[[0, 1, 3]]).all() and float((y[6] - 1).abs().max()) < 16 * U32
    _, (codes, scales) = sp.sp_rms_norm_q8(x, gamma)
    s = scales.view(torch.uint8)[:, 0].tolist()
    assert s[2] == 255 and s[4] == 255 and s[5] == 127 and not codes.view(torch.uint8)[5].any() and 255 not in (s[0], s[1], s[3], s[6])
    for bad in (lambda: sp.sp_rms_norm_fwd(x, gamma[:40]), lambda: sp.sp_rms_norm_fwd(x[:, ::2], gamma[:24].contiguous()),
                lambda: sp.sp_rms_norm_fwd(x, gamma, x[:3]), lambda: sp.sp_rms_norm_fwd(x, gamma, x.bfloat16()), lambda: sp.sp_rms_norm_fwd(x[0], gamma),
                lambda: sp.sp_rms_norm_q8(x, gamma.cpu()), lambda: sp.sp_rms_norm_bwd(x, y[:3], gamma, rstd), lambda: sp.sp_rms_norm_bwd(x, y, gamma, rstd[:3])):
        with pytest.raises(ValueError):
            bad()
    # rows off a 16-byte border take unaligned loads: the same lanes, the same bits
    flat = torch.randn(6 * 48 + 1, device="cuda")
    a, b = (sp.sp_rms_norm_fwd(t.view(6, 48), gamma)[1] for t in (flat[1:], flat[1:].clone()))
    assert torch.equal(a, b)


# ---- rows in 8 bits --------------------------------------------------------------------------------------------
def same_codes(got, want):
    assert np.array_equal(got[0].view(torch.uint8).cpu().numpy(), want[0]) and np.array_equal(got[1].view(torch.uint8).cpu().numpy(), want[1])


@TYPES
@pytest.mark.parametrize("n,c", [(1, 1), (3, 7), (5, 128), (129, 127), (256, 130), (17, 513), (300, 70), (1, 1024), (700, 3)])
def test_q8_rows(sp, n, c, dt):
    rng = np.random.default_rng(n + 3 * c)
    x = torch.from_numpy((rng.standard_normal((n, c)) * 2.0 ** rng.integers(-30, 30, (n, c))).astype(np.float32)).to(dt).cuda()
    same_codes(sp.sp_q8_rows(x), block.q8_rows(host(x)))
    same_codes(sp.sp_q8_rows(x, transposed=True), block.q8_rows(host(x).T))
    wide = rows(rng, dt, n, c + 5)
    same_codes(sp.sp_q8_rows(wide[:, 2:c + 2]), block.q8_rows(host(wide)[:, 2:c + 2]))
    same_codes(sp.sp_q8_rows(wide[:, 2:c + 2], transposed=True), block.q8_rows(host(wide)[:, 2:c + 2].T))


def test_q8_rows_of_every_kind_of_value(sp):
    x = torch.zeros((8, 256), device="cuda")
    x[0, 3], x[1, 200], x[2, 5] = float("inf"), float("-inf"), float("nan")
    x[3, :100] = torch.linspace(-448, 448, 100, device="cuda")
    x[4] = torch.ldexp(torch.randn(256, device="cuda"), torch.tensor(-130, device="cuda"))   # subnormal
    x[5, 0], x[5, 1] = torch.finfo(F32).max, -torch.finfo(F32).max
    x[6, 0], x[6, 128] = 448.0, 448.0001
    x[7] = -0.0
    same_codes(sp.sp_q8_rows(x), block.q8_rows(host(x)))
    same_codes(sp.sp_q8_rows(x, transposed=True), block.q8_rows(host(x).T))
    assert sp.sp_q8_rows(x[:0])[0].shape == (0, 256)
    for bad in (lambda: sp.sp_q8_rows(x.t()), lambda: sp.sp_q8_rows(x.half()), lambda: sp.sp_q8_rows(x.cpu()), lambda: sp.sp_q8_rows(x[0]),
                lambda: sp.sp_q8_rows(x[:0], transposed=True)):
        with pytest.raises(ValueError):
            bad()


def q8_bound(X, W, Y, out):
    """fp32 sums in some order: one rounding an element.  bf16 results come from 8-bit products.  These take eight neighbouring elements at a time and
    cut their products off at 2^-13 of the power of two in the largest: seven lose less than 2^-13 of the largest each, 7 * 2^-13 of it together,
    and it is no more than the eight's sizes' sum.  Then the result is rounded once."""
    size = np.abs(X) @ np.abs(W).T
    if out == F32:
        return (X.shape[1] + 70) * U32 * size
    lost = (7 * 2.0 ** -13 + (X.shape[1] + 70) * U32) * size
    return lost + half_step(BF16) * (np.abs(Y) + lost)


LINEAR = [(1, 1, 1), (1, 128, 4), (3, 70, 5), (32, 300, 130), (33, 128, 257), (40, 1000, 64), (128, 129, 128), (200, 640, 63), (300, 520, 500), (7, 4096, 33),
          (2, 8192, 300), (1100, 128, 1000), (513, 256, 770), (64, 5000, 65)]


@pytest.mark.parametrize("out", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,c,m", LINEAR)
def test_q8_linear(sp, n, c, m, out):
    rng = np.random.default_rng(n + c + m)
    spread = lambda k: torch.from_numpy(2.0 ** rng.integers(-6, 6, (k, c)).astype(np.float32)).cuda()  # noqa: E731
    x, w = rows(rng, F32, n, c) * spread(n), rows(rng, F32, m, c) * spread(m)
    qx, qw = sp.sp_q8_rows(x), sp.sp_q8_rows(w)
    X, W = (block.q8_values(q.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy()) for q, s in (qx, qw))
    y = sp.sp_q8_linear(qx, qw, out)
    Y = X @ W.T
    within(y, Y, q8_bound(X, W, Y, out), "y")
    assert y.dtype == out and torch.equal(y, sp.sp_q8_linear(qx, qw, out))


@pytest.mark.parametrize("out", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 70])
def test_q8_linear_of_extreme_scales(sp, n, out):
    rng = np.random.default_rng(n)
    x, w = rows(rng, F32, n, 256), rows(rng, F32, 40, 256)
    x[0] *= 2.0 ** 60
    x[1] *= 2.0 ** -60
    w[0] *= 2.0 ** 60
    w[1] *= 2.0 ** -60
    x[2, 5], w[3, 200] = float("nan"), float("inf")
    qx, qw = sp.sp_q8_rows(x), sp.sp_q8_rows(w)
    X, W = (block.q8_values(q.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy()) for q, s in (qx, qw))
    with np.errstate(invalid="ignore"):
        Y = X @ W.T
    y = sp.sp_q8_linear(qx, qw, out)
    assert torch.isnan(y[2]).all() and torch.isnan(y[:, 3]).all()
    within(y, Y, np.where(np.isfinite(Y), q8_bound(X, W, Y, out), 0), "y")


def test_q8_linear_refuses(sp):
    x = torch.randn((4, 200), device="cuda")
    q = sp.sp_q8_rows(x)
    other = sp.sp_q8_rows(x[:, :100].contiguous())
    for bad in (lambda: sp.sp_q8_linear(q, other), lambda: sp.sp_q8_linear(q, (q[0], q[1][:2])), lambda: sp.sp_q8_linear(q, (q[0].view(torch.uint8), q[1])),
                lambda: sp.sp_q8_linear(q, (q[0], q[1].view(torch.uint8))), lambda: sp.sp_q8_linear(q, q, torch.float16),
                lambda: sp.sp_q8_linear((q[0][:, :100].contiguous(), q[1]), q), lambda: sp.sp_q8_linear((q[0].cpu(), q[1]), q)):
        with pytest.raises(ValueError):
            bad()
    assert sp.sp_q8_linear((q[0][:0], q[1][:0]), q).shape == (0, 4)


@TYPES
def test_gradients_in_8_bits(sp, dt):
    """dx = dy w and dw = dy^T x from operands in 8 bits along the other axis: against the definition on what the codes stand for, and against
    the exact gradient within the codes' rounding (2^-4 of either operand's element, or 2^-10 of its block's scale)."""
    rng = np.random.default_rng(8)
    n, c, m = 150, 200, 90
    x, w, dy = rows(rng, dt, n, c), rows(rng, dt, m, c), rows(rng, dt, n, m)
    for a, b, ta, tb in ((dy, w, False, True), (dy, x, True, True)):
        qa, qb = sp.sp_q8_rows(a, transposed=ta), sp.sp_q8_rows(b, transposed=tb)
        A, B = (block.q8_values(q.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy()) for q, s in (qa, qb))
        got = sp.sp_q8_linear(qa, qb, dt)
        Y = A @ B.T
        within(got, Y, q8_bound(A, B, Y, dt), "gradient")
        EA, EB = (host(t).T if turned else host(t) for t, turned in ((a, ta), (b, tb)))
        off = lambda e: np.abs(e) / 16 + np.abs(e).max() / 448 * 2 / 1024  # noqa: E731
        slack = off(EA) @ np.abs(EB).T + np.abs(EA) @ off(EB).T + off(EA) @ off(EB).T
        assert (np.abs(Y - EA @ EB.T) <= slack).all()


# ---- gated feed-forward block ----------------------------------------------------------------------------------
# rows, width, hidden width
FFN = [(1, 1, 1), (1, 64, 64), (3, 5, 7), (31, 72, 136), (32, 128, 64), (33, 64, 129), (65, 71, 137), (130, 100, 270), (257, 64, 128), (300, 256, 260),
       (5, 1000, 520), (2, 520, 3000), (700, 16, 8), (129, 520, 512), (1025, 24, 40), (17, 2048, 96)]


def ffn_forward_bounds(X, WI, WO, act, u):
    """(bound of g and u, of h, of y): products and sums of the contraction's length; the gate's slope is below 1.13, its own error (an exponential or
    error function of a few steps) below 6 U32 |g|; results rounded to the storage type."""
    m, c = WO.shape[1], X.shape[1]
    Y, G, U, H = block.ffn_fwd(X, WI, WO, act)
    e = (c + 4) * U32 * (np.abs(X) @ np.abs(WI).T)
    eg, eu = e[:, :m], e[:, m:]
    a = block.gate(G, act)[0]
    ea = 1.13 * eg + 6 * U32 * np.abs(G)
    eh = ea * np.abs(U) + np.abs(a) * eu + ea * eu + 2 * U32 * np.abs(H)
    eh = eh + u * (np.abs(H) + eh)
    ey = eh @ np.abs(WO).T + (m + 4) * U32 * ((np.abs(H) + eh) @ np.abs(WO).T)
    cut = 2.0 ** -15 if u > U32 else U32                     # g and u are kept in 24 bits of fp32, cut off
    return (Y, G, U, H), (e + cut * (np.abs(np.concatenate([G, U], 1)) + e), eh, ey + u * (np.abs(Y) + ey))


def kept_values(kept, m):
    """[g u h] as the backward pass takes them: in bf16 g and u have 8 more bits in a fourth part."""
    if kept.dtype == F32:
        return host(kept)
    bits = kept.to(torch.int32) & 0xffff
    g, u, lo = bits[:, :m], bits[:, m:2 * m], bits[:, 3 * m:]
    g, u = (g << 16) | ((lo & 255) << 8), (u << 16) | (lo & 0xff00)
    return np.concatenate([host(g.view(F32)), host(u.view(F32)), host(kept[:, 2 * m:3 * m].contiguous().view(BF16))], 1)


def ffn_backward_bounds(X, WI, WO, kept, DY, act, u):
    m, c, n = WO.shape[1], X.shape[1], X.shape[0]
    G, U, H = kept[:, :m], kept[:, m:2 * m], kept[:, 2 * m:]
    dx, dwi, dwo, dgu = block.ffn_bwd(X, WI, WO, G, U, H, DY, act)
    a, da = block.gate(G, act)
    dh = DY @ WO
    e = (c + 4) * U32 * (np.abs(DY) @ np.abs(WO))
    ea, eda = 6 * U32 * np.abs(G), 8 * U32 * (1 + np.abs(G))
    eg = (e * np.abs(da) + (np.abs(dh) + e) * eda) * np.abs(U) + 3 * U32 * np.abs(dgu[:, :m])
    eu = e * np.abs(a) + (np.abs(dh) + e) * ea + 3 * U32 * np.abs(dgu[:, m:])
    ed = np.concatenate([eg, eu], 1)
    ed = ed + u * (np.abs(dgu) + ed)
    big = np.abs(dgu) + ed

    def last(v, err, *sizes):
        err = err + sum(sizes)
        return err + u * (np.abs(v) + err)

    return (dx, dwi, dwo), (last(dx, ed @ np.abs(WI), (2 * m + 4) * U32 * (big @ np.abs(WI))), last(dwi, ed.T @ np.abs(X), (n + 70) * U32 * (big.T @ np.abs(X))),
                            last(dwo, 0, (n + 70) * U32 * (np.abs(DY).T @ np.abs(H))))


@TYPES
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,c,m", FFN)
def test_ffn(sp, n, c, m, act, dt):
    rng = np.random.default_rng(n + c + m)
    x, dy = rows(rng, dt, n, c), rows(rng, dt, n, c)
    w_in, w_out = rows(rng, dt, 2 * m, c, scale=1.5 / math.sqrt(c)), rows(rng, dt, c, m, scale=1 / math.sqrt(m))
    u = half_step(dt) if dt == BF16 else U32
    X, DY, WI, WO = host(x), host(dy), host(w_in), host(w_out)
    (Y, G, U, H), (e_gu, e_h, e_y) = ffn_forward_bounds(X, WI, WO, act, u)
    y, kept = sp.sp_ffn_fwd(x, w_in, w_out, act)
    within_values(kept_values(kept, m), np.concatenate([G, U, H], 1), np.concatenate([e_gu, e_h], 1), "kept")
    within(y, Y, e_y, "y")
    alone = sp.sp_ffn_fwd(x, w_in, w_out, act, keep=False)
    assert torch.equal(alone, y)
    grads = sp.sp_ffn_bwd(x, w_in, w_out, kept, dy, act)
    want, bounds = ffn_backward_bounds(X, WI, WO, kept_values(kept, m), DY, act, u)
    for got, ref, bound, name in zip(grads, want, bounds, ("dx", "dw_in", "dw_out")):
        assert got.dtype == dt
        within(got, ref, bound, name)
    again = sp.sp_ffn_bwd(x, w_in, w_out, kept, dy, act)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@TYPES
def test_ffn_edges(sp, dt):
    w_in, w_out = torch.randn((48, 40), device="cuda").to(dt), torch.randn((40, 24), device="cuda").to(dt)
    empty = torch.empty((0, 40), device="cuda", dtype=dt)
    y, kept = sp.sp_ffn_fwd(empty, w_in, w_out)
    dx, dw_in, dw_out = sp.sp_ffn_bwd(empty, w_in, w_out, kept, empty)
    assert y.shape == dx.shape == (0, 40) and not dw_in.any() and not dw_out.any()
    x = torch.randn((9, 40), device="cuda").to(dt)
    x[4, 7] = float("nan")
    y = sp.sp_ffn_fwd(x, w_in, w_out, keep=False)
    assert torch.isnan(y[4]).all() and torch.isfinite(y[[0, 1, 2, 3, 5, 6, 7, 8]]).all()
    flat = torch.randn(9 * 40 + 1, device="cuda").to(dt)     # off a 16-byte border: through registers, in the same order
    assert torch.equal(sp.sp_ffn_fwd(flat[1:].view(9, 40), w_in, w_out, keep=False), sp.sp_ffn_fwd(flat[1:].clone().view(9, 40), w_in, w_out, keep=False))
    x = torch.randn((9, 40), device="cuda").to(dt)
    y, kept = sp.sp_ffn_fwd(x, w_in, w_out)
    for bad in (lambda: sp.sp_ffn_fwd(x, w_in[:40], w_out), lambda: sp.sp_ffn_fwd(x, w_in, w_out.t()), lambda: sp.sp_ffn_fwd(x, w_in, w_out, act="relu"),
                lambda: sp.sp_ffn_fwd(x[:, :39], w_in, w_out), lambda: sp.sp_ffn_fwd(x, w_in.half(), w_out), lambda: sp.sp_ffn_fwd(x[0], w_in, w_out),
                lambda: sp.sp_ffn_bwd(x, w_in, w_out, kept[:, :48].contiguous(), y), lambda: sp.sp_ffn_bwd(x, w_in, w_out, kept, y[:3])):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_ffn_gates_of_large_values(sp, act):
    """Far from zero a gate is its argument or nothing, and its slope 1 or 0."""
    g = torch.tensor([-1e4, -200.0, -100.0, 100.0, 200.0, 1e4], device="cuda")[:, None]
    w_in, w_out = torch.tensor([[1.0], [0.0]], device="cuda"), torch.ones((1, 1), device="cuda")
    _, kept = sp.sp_ffn_fwd(g, w_in, w_out, act)
    assert torch.isfinite(kept).all()
    kept[:, 1] = 2.0                                         # u, in fp32
    dx, _, _ = sp.sp_ffn_bwd(g, w_in, w_out, kept, torch.ones_like(g), act)
    assert torch.equal(dx[3:, 0], torch.full((3,), 2.0, device="cuda")) and float(dx[:3].abs().max()) < 1e-30


# ---- larger products: every workgroup's shape, split and joined --------------------------------------------------
@pytest.mark.parametrize("n,c,m,dt", [(4096, 512, 1024, BF16), (3000, 1032, 520, BF16), (1500, 264, 300, F32), (24, 2048, 4096, BF16), (20000, 64, 96, BF16),
                                      (2100, 1024, 1024, F32), (600, 500, 1000, BF16)])
def test_large_ffn_by_samples(sp, n, c, m, dt):
    """Some rows and columns of every result, against the definition."""
    g = torch.Generator(device="cuda").manual_seed(n)
    normal = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    x, dy = normal(n, c).to(dt), normal(n, c).to(dt)
    w_in, w_out = (normal(2 * m, c) / math.sqrt(c)).to(dt), (normal(c, m) / math.sqrt(m)).to(dt)
    u = half_step(dt) if dt == BF16 else U32
    y, kept = sp.sp_ffn_fwd(x, w_in, w_out, "silu")
    r = torch.unique(torch.cat([torch.randint(0, n, (40,), generator=torch.Generator().manual_seed(1)), torch.tensor([0, n - 1])])).cuda()
    X, WI, WO = host(x[r]), host(w_in), host(w_out)
    (Y, G, U, H), (e_gu, e_h, e_y) = ffn_forward_bounds(X, WI, WO, "silu", u)
    within_values(kept_values(kept[r], m), np.concatenate([G, U, H], 1), np.concatenate([e_gu, e_h], 1), "kept")
    within(y[r], Y, e_y, "y")
    dx, dw_in, dw_out = sp.sp_ffn_bwd(x, w_in, w_out, kept, dy, "silu")
    (DX, _, _), (e_dx, _, _) = ffn_backward_bounds(X, WI, WO, kept_values(kept[r], m), host(dy[r]), "silu", u)
    within(dx[r], DX, e_dx, "dx")
    # some hidden channels' weights: their columns of dgu, all rows
    j = torch.unique(torch.cat([torch.randint(0, m, (20,), generator=torch.Generator().manual_seed(2)), torch.tensor([0, m - 1])])).cuda()
    cols = j.cpu().numpy()
    k = kept_values(kept, m)[:, np.concatenate([cols, m + cols, 2 * m + cols])]
    (_, DWI, DWO), (_, e_wi, e_wo) = ffn_backward_bounds(host(x), host(torch.cat([w_in[j], w_in[m + j]])), host(w_out[:, j]), k, host(dy), "silu", u)
    within(torch.cat([dw_in[j], dw_in[m + j]]), DWI, e_wi, "dw_in")
    within(dw_out[:, j], DWO, e_wo, "dw_out")


@pytest.mark.parametrize("n,c,m", [(2000, 1024, 1536), (5000, 640, 1000), (31, 4096, 6144), (260, 8192, 512)])
def test_large_q8_linear_by_samples(sp, n, c, m):
    g = torch.Generator(device="cuda").manual_seed(n)
    qx, qw = (sp.sp_q8_rows(torch.randn((k, c), device="cuda", generator=g)) for k in (n, m))
    r = torch.unique(torch.cat([torch.randint(0, n, (60,), generator=torch.Generator().manual_seed(1)), torch.tensor([0, n - 1])])).cuda()
    X, W = (block.q8_values(q.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy())
            for q, s in ((qx[0].view(torch.uint8)[r], qx[1].view(torch.uint8)[r]), qw))
    Y = X @ W.T
    for out in (F32, BF16):
        within(sp.sp_q8_linear(qx, qw, out)[r], Y, q8_bound(X, W, Y, out), "y")


# ---- streams and graphs ----------------------------------------------------------------------------------------
def every_operator(sp, s):
    """All operators in a row, as a block would use them; returns what they give."""
    turn = dict(parts=(12, 10, 10), split=True)
    h, n1, rstd = sp.sp_rms_norm_fwd(s["x"], s["gamma"], s["res"])
    q = sp.sp_rope_fwd(n1.view(-1, 3, 32), s["pos"], **turn)
    y, kept = sp.sp_ffn_fwd(n1, s["w_in"], s["w_out"])
    dn, dwi, dwo = sp.sp_ffn_bwd(n1, s["w_in"], s["w_out"], kept, s["dy"])
    dq = sp.sp_rope_bwd(dn.view(-1, 3, 32), s["pos"], **turn)
    dx, dgamma = sp.sp_rms_norm_bwd(h, dn, s["gamma"], rstd, dq.view(-1, 96))
    _, q8 = sp.sp_rms_norm_q8(y, s["gamma"], h)
    z = sp.sp_q8_linear(q8, sp.sp_q8_rows(s["w_in"]))
    t = sp.sp_q8_linear(sp.sp_q8_rows(s["dy"], transposed=True), sp.sp_q8_rows(n1, transposed=True), torch.float32)
    return [h, n1, rstd, q, y, kept, dn, dwi, dwo, dq, dx, dgamma, z, t]


def block_state(seed, n):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    return {"x": normal(n, 96).bfloat16(), "res": normal(n, 96).bfloat16(), "dy": normal(n, 96).bfloat16(), "gamma": 1 + 0.1 * normal(96),
            "w_in": (normal(400, 96) / 10).bfloat16(), "w_out": (normal(96, 200) / 14).bfloat16(),
            "pos": torch.randint(-300, 300, (n, 3), dtype=torch.int32, device="cuda", generator=g)}


def test_two_captured_graphs_and_eager_work_between(sp):
    """Each graph has work memory of its own: replays of both, with eager calls of other sizes between them, give the eager results every time."""
    states = [block_state(1, 700), block_state(2, 9)]
    want = [[t.clone() for t in every_operator(sp, s)] for s in states]
    graphs, outs = [], []
    for s in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(every_operator(sp, s))
        graphs.append(graph)
    other = block_state(3, 333)
    first = [t.clone() for t in every_operator(sp, other)]
    for turn in range(4):
        for graph in graphs:
            graph.replay()
        again = every_operator(sp, other)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
        if turn % 2:
            torch.cuda.synchronize()
        for got, ref in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(got, ref)), turn
        for o in outs:
            for t in o:
                t.zero_()


def test_two_streams_at_once(sp):
    states = [block_state(4, 2000), block_state(5, 1500)]
    want = [[t.clone() for t in every_operator(sp, s)] for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, stream in zip(states, streams):
            with torch.cuda.stream(stream):
                got.append(every_operator(sp, s))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---- rows that end inside a load, small matrices in one launch, gates of every size --------------------------------
@TYPES
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,c,m", [(200, 3, 5), (400, 6, 10), (333, 7, 9), (2049, 33, 70), (600, 1030, 24), (96, 4, 2050), (40, 952, 330), (3000, 100, 270)])
def test_ffn_of_rows_that_end_inside_a_load(sp, n, c, m, act, dt):
    """Contractions of several steps over rows of no whole 16 bytes, down to rows shorter than a load."""
    test_ffn(sp, n, c, m, act, dt)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n", [7, 4000])
def test_gates_over_their_range(sp, act, n):
    """u = 1, W_out = 1: y is act(g), rounded once; its own error is below 6 U32 |g|.  dx (dy = 1, W_in = (1, 0; 0, 1)) is (act'(g), act(g)) as dgu is
    rounded: the slope's error is below 8 U32 (1 + |g|)."""
    g = torch.linspace(-12, 12, n, device="cuda").bfloat16()
    x = torch.stack([g, torch.ones_like(g)], 1)
    w_in, w_out = torch.eye(2, device="cuda").bfloat16(), torch.tensor([[1.0], [0.0]], device="cuda").bfloat16()
    y, kept = sp.sp_ffn_fwd(x, w_in, w_out, act)
    G = host(g)
    a, da = block.gate(G, act)
    u = half_step(BF16)
    err = 6 * U32 * np.abs(G)
    within(y[:, 0], a, err + u * (np.abs(a) + err), "act")
    dx, _, _ = sp.sp_ffn_bwd(x, w_in, w_out, kept, torch.ones_like(x), act)
    err = 8 * U32 * (1 + np.abs(G))
    within(dx[:, 0], da, err + u * (np.abs(da) + err), "slope")


@TYPES
@pytest.mark.parametrize("n,c", [(1428, 128), (60, 77), (4096, 64), (4097, 64), (900, 1024), (3, 16392)])
def test_rms_norm_gradients_in_place(sp, n, c, dt):
    """dx in dy's or dh's memory: the same results, in one launch or several."""
    rng = np.random.default_rng(n + c)
    h, dy, dh = (rows(rng, dt, n, c) for _ in range(3))
    gamma = 1 + rows(rng, F32, c, scale=0.2)
    rstd = 1 / torch.sqrt((h.float() ** 2).mean(1) + 1e-5)
    dx, dgamma = sp.sp_rms_norm_bwd(h, dy, gamma, rstd, dh)
    l = sp._block_argtypes()
    for which in (0, 1):
        a = [dy.clone(), dh.clone()]
        got, work = torch.empty_like(gamma), torch.empty(l.sp_rms_norm_bwd_work(n, c, sp._dt(h)), dtype=torch.uint8, device="cuda")
        assert l.sp_rms_norm_bwd(h.data_ptr(), a[0].data_ptr(), a[1].data_ptr(), n, c, gamma.data_ptr(), rstd.data_ptr(), a[which].data_ptr(),
                                 got.data_ptr(), work.data_ptr(), sp._dt(h), sp._stream()) == 0
        assert torch.equal(a[which], dx) and torch.equal(got, dgamma)


@pytest.mark.parametrize("n,c,m", [(32, 640, 77), (33, 640, 77), (70, 3000, 40), (300, 12800, 24), (1, 12900, 9), (129, 130, 260)])
def test_q8_linear_of_many_steps(sp, n, c, m):
    """Four steps share a word of scales, and parts begin at one: scales that differ from step to step."""
    g = torch.Generator(device="cuda").manual_seed(n + c)
    grow = lambda k: torch.randn((k, c), device="cuda", generator=g) * 2.0 ** torch.randint(-6, 6, (k, -(-c // 128)), device="cuda", generator=g).float().repeat_interleave(128, 1)[:, :c]  # noqa: E731
    (x, xs), (w, ws) = sp.sp_q8_rows(grow(n)), sp.sp_q8_rows(grow(m))
    X, W = (block.q8_values(q.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy()) for q, s in ((x, xs), (w, ws)))
    Y = X @ W.T
    for out in (F32, BF16):
        within(sp.sp_q8_linear((x, xs), (w, ws), out), Y, q8_bound(X, W, Y, out), "y")


@pytest.mark.parametrize("n,c,m", [(600, 504, 1000), (700, 768, 3000), (6000, 256, 512), (300, 1024, 4096), (1697, 512, 1024)])
def test_ffn_of_a_workgroup_a_cu(sp, n, c, m):
    """Fewer workgroups than CUs, in one part and in several: the deeper tiles."""
    test_large_ffn_by_samples(sp, n, c, m, BF16)


@pytest.mark.parametrize("n,c,m", [(2048, 2048, 2048), (1000, 4096, 1024), (1500, 1800, 1900)])
def test_q8_linear_of_a_workgroup_a_cu(sp, n, c, m):
    test_large_q8_linear_by_samples(sp, n, c, m)


@TYPES
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,c,m", [(32, 136, 256), (32, 64, 128), (32, 512, 1024), (31, 136, 256)])
def test_ffn_of_a_tile_of_32_rows(sp, n, c, m, act, dt):
    """Tiles of 128 x 32 that lie within the results: the gradient's last step has two items a lane, and reads no more of them ahead."""
    test_ffn(sp, n, c, m, act, dt)


@TYPES
@pytest.mark.parametrize("c", [1, 77, 4096, 8192, 16392, 65536])
def test_rms_norm_of_the_largest_values(sp, c, dt):
    """Squares beyond fp32, whatever the width; rstd is then below 2^-126, where fp32 has steps of 2^-149."""
    rng = np.random.default_rng(c)
    x = torch.from_numpy((rng.uniform(1e38, 3.3e38, (3, c)) * rng.choice([-1, 1], (3, c))).astype(np.float32)).to(dt).cuda()
    gamma = 1 + rows(rng, F32, c, scale=0.2)
    _, y, rstd = sp.sp_rms_norm_fwd(x, gamma)
    Y, R = block.rms_fwd(host(x), host(gamma), 1e-5)
    rel = sum_error(c) / 2 + 4 * U32
    within(rstd, R, rel * R + 2.0 ** -150, "rstd")
    within(y, Y, (rel + 3 * U32 + half_step(dt) + 2.0 ** -150 / R.min()) * np.abs(Y), "y")
    _, q8 = sp.sp_rms_norm_q8(x, gamma)
    V = block.q8_values(*(t.view(torch.uint8).cpu().numpy() for t in q8))[:, :c]
    err = (rel + 3 * U32 + 2.0 ** -150 / R.min()) * np.abs(Y)
    # half a step of a code: 2^-4 of the value, or of the smallest step, 2^-9 of a scale that is below 2^-7 of the block's largest element
    assert (np.abs(V - Y) <= err + np.maximum((np.abs(Y) + err) / 16, np.abs(Y).max() * 2.0 ** -17)).all()


@TYPES
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-32])
@pytest.mark.parametrize("c", [1, 13, 128, 1000, 4096, 16392])
def test_rms_norm_of_small_values(sp, c, eps, dt):
    """Squares that underflow, beside an eps that does not cover them: the definition all the same, rstd as far as fp32 goes."""
    rng = np.random.default_rng(c)
    sizes = np.array([1e-10, 1e-15, 1e-17, 1e-19, 1e-21, 1e-24, 1e-30, 1e-36, 1e-39, 0.0])[:, None]
    x = torch.from_numpy((rng.uniform(0.5, 2, (10, c)) * rng.choice([-1, 1], (10, c)) * sizes).astype(np.float32)).to(dt).cuda()
    dy = rows(rng, dt, 10, c)
    gamma = 1 + rows(rng, F32, c, scale=0.2)
    exact = float(np.float32(eps))
    _, y, rstd = sp.sp_rms_norm_fwd(x, gamma, eps=eps)
    with np.errstate(divide="ignore", invalid="ignore"):
        Y, R = block.rms_fwd(host(x), host(gamma), exact)
    assert torch.isnan(y[9]).all() if eps == 0 else not y[9].any()
    rel = sum_error(c) / 2 + 4 * U32
    within(rstd, np.where(R > 2.0 ** 128, np.inf, R), rel * R, "rstd")
    within(y, Y, (rel + 3 * U32 + half_step(dt)) * np.abs(Y), "y")
    _, q8 = sp.sp_rms_norm_q8(x, gamma, eps=eps)
    V = block.q8_values(*(t.view(torch.uint8).cpu().numpy() for t in q8))[:9, :c]
    err = (rel + 3 * U32) * np.abs(Y[:9])
    # half a step of a code: 2^-4 of the value, or of the smallest step, 2^-9 of a scale that is below 2^-7 of the block's largest element
    assert (np.abs(V - Y[:9]) <= err + np.maximum((np.abs(Y[:9]) + err) / 16, np.abs(Y[:9]).max(1, keepdims=True) * 2.0 ** -17)).all()
    # gradients of the rows that have an rstd, from the GPU's own, where they are within fp32
    live = slice(0, 6)
    dx, dgamma = sp.sp_rms_norm_bwd(x[live].contiguous(), dy[live].contiguous(), gamma, rstd[live].contiguous())
    H, D, S = host(x[live]), host(dy[live]), host(rstd[live])
    DX, DG = block.rms_bwd(H, D, host(gamma), S)
    hat, g = np.abs(H * S[:, None]), np.abs(D * host(gamma))
    size = S[:, None] * (g + hat * (g * hat).mean(1)[:, None])
    within(dx, DX, (sum_error(c) + 6 * U32) * size + (half_step(dt) + U32) * np.abs(DX), "dx")
    within(dgamma, DG, 18 * U32 * np.abs(D * hat).sum(0) + U32 * np.abs(DG), "dgamma")


@pytest.mark.parametrize("n", [7, 4000])
def test_gelu_keeps_its_tail_in_fp32(sp, n):
    """u = 1, W_out = 1: y is gelu(g) = g p, dx its slope p + g f (p the normal distribution function, f its density).  erfc is within 16 steps of fp32 (32 U32) of
    an argument rounded twice, which moves it by 2 U32 g^2 of itself; the exponential in f within 8 U32 of an argument rounded twice, g^2 U32 of it."""
    g = torch.linspace(-12.5, 12.5, n, device="cuda")
    x = torch.stack([g, torch.ones_like(g)], 1)
    w_in, w_out = torch.eye(2, device="cuda"), torch.tensor([[1.0], [0.0]], device="cuda")
    y, kept = sp.sp_ffn_fwd(x, w_in, w_out, "gelu")
    G = host(g)
    p, f = np.array([math.erfc(-v / math.sqrt(2)) / 2 for v in G]), np.exp(-G * G / 2) / math.sqrt(2 * math.pi)
    within(y[:, 0], G * p, (36 + 2 * G * G) * U32 * np.abs(G) * p, "gelu")
    dx, _, _ = sp.sp_ffn_bwd(x, w_in, w_out, kept, torch.ones_like(x), "gelu")
    within(dx[:, 0], p + G * f, U32 * ((36 + 2 * G * G) * p + (12 + 2 * G * G) * np.abs(G) * f), "slope")


@pytest.mark.parametrize("out", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,c,m", [(9, 100, 20), (9, 1300, 40), (70, 640, 150), (300, 200, 90)])
def test_q8_linear_of_scales_over_their_range(sp, n, c, m, out):
    """Rows from subnormal to the largest values, codes of every scale that there is.  Compared where the products' sizes sum to less than 2^127 and, of the scaled
    instruction (bf16), to more than 2^-100; elsewhere a result may be infinite, or below what fp32 holds.  Each step's sum may be subnormal: half of 2^-149."""
    rng = np.random.default_rng(n + c)
    x, w = rows(rng, F32, n, c), rows(rng, F32, m, c)
    for t, sizes in ((x, (-145, -133, -126, -118, -100, 0, 60, 120)), (w, (-140, -127, -120, -60, -35, -10, 0, 10, 100, 120))):
        for r in range(t.shape[0]):
            t[r] = torch.ldexp(t[r], torch.tensor(sizes[r % len(sizes)], device="cuda"))
    x[4] = torch.where(x[4] > 0, 3.39e38, -3.39e38)          # 256 times 2^120: beyond bf16
    w[5, :50] = 0
    w[6] = 0
    qx, qw = sp.sp_q8_rows(x), sp.sp_q8_rows(w)
    s = qx[1].view(torch.uint8)
    s[n - 1, 0], s[n - 2, 0] = 254, 1                        # larger ones than any row's own
    X, W = (block.q8_values(q.view(torch.uint8).cpu().numpy(), e.view(torch.uint8).cpu().numpy()) for q, e in (qx, qw))
    size = np.abs(X) @ np.abs(W).T
    Y = X @ W.T
    y = sp.sp_q8_linear(qx, qw, out)
    seen = (size < 2.0 ** 127) & ((size > 2.0 ** -100) | (size == 0) if out == BF16 else True)
    assert seen.mean() > 0.3 and not y[:, 6].any()
    got = host(y)
    bound = q8_bound(X, W, Y, out) + -(-c // 128) * 2.0 ** -149
    within_values(np.where(seen, got, 0), np.where(seen, Y, 0), bound, "y")


# ---- more rows than one launch takes ---------------------------------------------------------------------------
def test_q8_rows_transposed_of_more_rows_than_a_launch_takes(sp):
    """2^31 + 77 rows of one element: every 2^29 of them by themselves have the same codes."""
    n, most = (1 << 31) + 77, 1 << 29
    x = torch.randn((most + 3, 1), device="cuda").bfloat16().repeat(5, 1)[:n]
    codes, scales = (t.view(torch.uint8) for t in sp.sp_q8_rows(x, transposed=True))
    for at in range(0, n, most):
        some = x[at:at + most]
        q, s = (t.view(torch.uint8) for t in sp.sp_q8_rows(some, transposed=True))
        blocks = -(-some.shape[0] // 128)
        assert torch.equal(codes[:, at:at + blocks * 128], q) and torch.equal(scales[:, at // 128:at // 128 + blocks], s[:, :blocks]), at
    assert (scales[:, -(-n // 128):] == 127).all()
    del x, codes, scales, some, q, s
    torch.cuda.empty_cache()


def test_q8_rows_transposed_of_the_widest(sp):
    """2^22 columns: the largest grid across."""
    x = torch.randn((3, 1 << 22), device="cuda").bfloat16()
    codes, scales = (t.view(torch.uint8) for t in sp.sp_q8_rows(x, transposed=True))
    for at in (0, (1 << 21) - 64, (1 << 22) - 200):
        q, s = (t.view(torch.uint8) for t in sp.sp_q8_rows(x[:, at:at + 200].contiguous(), transposed=True))
        assert torch.equal(codes[at:at + 200], q) and torch.equal(scales[at:at + 200], s)
    del x, codes, scales
    torch.cuda.empty_cache()


@pytest.mark.parametrize("split", [False, True], ids=["neighbours", "halves"])
def test_rope_of_more_rows_than_a_launch_takes(sp, split):
    """2^27 + 1000 rows of 256, eight rows a workgroup of 256 threads, in place: rows here and there by themselves turn to the same bits."""
    n = (1 << 27) + 1000
    x = torch.ones((n, 1, 256), dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[:, None]
    sp.sp_rope_fwd(x, pos, (256,), split=split, out=x)
    for at in (0, (1 << 25) - 500, (1 << 26) - 500, (1 << 27) - 500, n - 1000):
        want = sp.sp_rope_fwd(torch.ones((1000, 1, 256), dtype=torch.bfloat16, device="cuda"), pos[at:at + 1000], (256,), split=split)
        assert torch.equal(x[at:at + 1000], want), at
    del x, pos
    torch.cuda.empty_cache()


@pytest.mark.parametrize("out", [F32, BF16], ids=["f32", "bf16"])
def test_q8_linear_of_more_weights_than_a_launch_of_few_rows_takes(sp, out):
    """Few rows by 2^24 + 2^20 + 40 weights, 2^24 of them a launch: weights here and there by themselves give the same bits."""
    m = (1 << 24) + (1 << 20) + 40
    g = torch.Generator(device="cuda").manual_seed(5)
    qx = sp.sp_q8_rows(torch.randn((3, 100), device="cuda", generator=g))
    q, s = sp.sp_q8_rows(torch.randn((m, 100), device="cuda", generator=g))
    y = sp.sp_q8_linear(qx, (q, s), out)
    for at in (0, (1 << 23) - 100, (1 << 24) - 1000, m - 2000):
        assert torch.equal(y[:, at:at + 2000], sp.sp_q8_linear(qx, (q[at:at + 2000], s[at:at + 2000]), out)), at
    del q, s, y
    torch.cuda.empty_cache()


@TYPES
@pytest.mark.parametrize("n,c", [(1428, 128), (60, 77), (5000, 64), (9, 4096), (5, 8191), (3, 16392), (4, 40001)])
def test_rms_norm_forward_in_place(sp, n, c, dt):
    """The sum in x's or the residual's memory, y in either that the sum is not in (or in x, without a residual): the same bits."""
    rng = np.random.default_rng(n + c)
    x, res = rows(rng, dt, n, c), rows(rng, dt, n, c)
    gamma = 1 + rows(rng, F32, c, scale=0.2)
    l, t, stream = sp._block_argtypes(), sp._dt(x), sp._stream()
    h, y, rstd = sp.sp_rms_norm_fwd(x, gamma, res)
    _, (q, s) = sp.sp_rms_norm_q8(x, gamma, res)
    for sum_in, out_in in ((0, None), (1, None), (0, 1), (1, 0), (None, 0), (None, 1)):
        own = [x.clone(), res.clone()]
        to_h, to_y = own[sum_in] if sum_in is not None else torch.empty_like(x), own[out_in] if out_in is not None else torch.empty_like(x)
        r = torch.empty_like(rstd)
        assert l.sp_rms_norm_fwd(own[0].data_ptr(), own[1].data_ptr(), n, c, gamma.data_ptr(), 1e-5, to_h.data_ptr(), to_y.data_ptr(), r.data_ptr(), t, stream) == 0
        assert torch.equal(to_h, h) and torch.equal(to_y, y) and torch.equal(r, rstd), (sum_in, out_in)
        if out_in is None:
            own = [x.clone(), res.clone()]
            q2, s2 = sp._q8_new(n, c, x.device)
            assert l.sp_rms_norm_q8(own[0].data_ptr(), own[1].data_ptr(), n, c, gamma.data_ptr(), 1e-5, own[sum_in].data_ptr(), q2.data_ptr(), s2.data_ptr(), t, stream) == 0
            assert torch.equal(own[sum_in], h) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2.view(torch.uint8), s.view(torch.uint8))
    _, y, rstd = sp.sp_rms_norm_fwd(x, gamma)
    own, r = x.clone(), torch.empty_like(rstd)
    assert l.sp_rms_norm_fwd(own.data_ptr(), None, n, c, gamma.data_ptr(), 1e-5, None, own.data_ptr(), r.data_ptr(), t, stream) == 0
    assert torch.equal(own, y) and torch.equal(r, rstd)


# ---- memory beyond 32 bits of bytes, and off 16-byte borders -----------------------------------------------------
def off_border(t):
    """The same values one element behind a 16-byte border."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


@TYPES
@pytest.mark.parametrize("which", ["x", "w_in", "w_out", "dy", "kept", "all"])
@pytest.mark.parametrize("n,c,m", [(20, 64, 128), (500, 72, 136), (2000, 256, 512)])
def test_ffn_of_unaligned_memory(sp, n, c, m, which, dt):
    """Each array by itself off a border: its products alone go through registers."""
    rng = np.random.default_rng(n)
    t = {"x": rows(rng, dt, n, c), "dy": rows(rng, dt, n, c), "w_in": rows(rng, dt, 2 * m, c, scale=1.5 / math.sqrt(c)), "w_out": rows(rng, dt, c, m, scale=1 / math.sqrt(m))}
    t = {k: off_border(v) if which in (k, "all") else v for k, v in t.items()}
    u = half_step(dt) if dt == BF16 else U32
    X, DY, WI, WO = (host(t[k]) for k in ("x", "dy", "w_in", "w_out"))
    (Y, _, _, _), (_, _, e_y) = ffn_forward_bounds(X, WI, WO, "silu", u)
    y, kept = sp.sp_ffn_fwd(t["x"], t["w_in"], t["w_out"])
    within(y, Y, e_y, "y")
    if which in ("kept", "all"):
        kept = off_border(kept)
    want, bounds = ffn_backward_bounds(X, WI, WO, kept_values(kept, m), DY, "silu", u)
    for got, ref, bound, name in zip(sp.sp_ffn_bwd(t["x"], t["w_in"], t["w_out"], kept, t["dy"]), want, bounds, ("dx", "dw_in", "dw_out")):
        within(got, ref, bound, name)


def test_ffn_of_more_than_32_bits_of_bytes(sp):
    """What is kept of 300007 rows of 2048 gates is 4.9 GB: rows at both ends, and the weights' gradients of a few hidden channels."""
    n, c, m, u = 300007, 64, 2048, half_step(BF16)
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    x, dy = normal(n, c).bfloat16(), normal(n, c).bfloat16()
    w_in, w_out = (normal(2 * m, c) / 8).bfloat16(), (normal(c, m) / math.sqrt(m)).bfloat16()
    y, kept = sp.sp_ffn_fwd(x, w_in, w_out)
    dx, dw_in, dw_out = sp.sp_ffn_bwd(x, w_in, w_out, kept, dy)
    r = torch.tensor([0, 1, 131071, 262143, 262144, n - 130, n - 2, n - 1], device="cuda")
    WI, WO = host(w_in), host(w_out)
    (Y, _, _, _), (_, _, e_y) = ffn_forward_bounds(host(x[r]), WI, WO, "silu", u)
    within(y[r], Y, e_y, "y")
    (DX, _, _), (e_dx, _, _) = ffn_backward_bounds(host(x[r]), WI, WO, kept_values(kept[r], m), host(dy[r]), "silu", u)
    within(dx[r], DX, e_dx, "dx")
    j = torch.tensor([0, 777, m - 1], device="cuda")
    k = kept_values(kept[:, torch.cat([j, m + j, 2 * m + j, 3 * m + j])], 3)
    (_, DWI, DWO), (_, e_wi, e_wo) = ffn_backward_bounds(host(x), host(torch.cat([w_in[j], w_in[m + j]])), host(w_out[:, j]), k, host(dy), "silu", u)
    within(torch.cat([dw_in[j], dw_in[m + j]]), DWI, e_wi, "dw_in")
    within(dw_out[:, j], DWO, e_wo, "dw_out")
    del x, y, dx, dy, kept
    torch.cuda.empty_cache()


def test_norm_and_rows_in_8_bits_of_more_than_32_bits_of_bytes(sp):
    """4.9 GB of rows, 2.5 GB of codes: the last rows by themselves give the same bits, and the product of the codes is the definition's."""
    n, c = 300007, 8192
    gamma = 1 + 0.1 * torch.randn(c, device="cuda")
    x = torch.empty((n, c), dtype=BF16, device="cuda").normal_()
    dy = x.flip(0)
    _, y, rstd = sp.sp_rms_norm_fwd(x, gamma)
    dx, _ = sp.sp_rms_norm_bwd(x, dy, gamma, rstd)
    _, (q, s) = sp.sp_rms_norm_q8(x, gamma)
    for at in (0, 262140, n - 300):
        some = x[at:at + 300].contiguous()
        _, ys, rs = sp.sp_rms_norm_fwd(some, gamma)
        assert torch.equal(ys, y[at:at + 300]) and torch.equal(rs, rstd[at:at + 300])
        assert torch.equal(sp.sp_rms_norm_bwd(some, dy[at:at + 300].contiguous(), gamma, rs)[0], dx[at:at + 300])
        qs, ss = sp.sp_rms_norm_q8(some, gamma)[1]
        assert torch.equal(qs.view(torch.uint8), q[at:at + 300].view(torch.uint8)) and torch.equal(ss.view(torch.uint8), s[at:at + 300].view(torch.uint8))
        assert all(torch.equal(a.view(torch.uint8), b[at:at + 300].view(torch.uint8)) for a, b in zip(sp.sp_q8_rows(ys), sp.sp_q8_rows(y)))
    del x, y, dx, dy
    torch.cuda.empty_cache()
    wq = sp.sp_q8_rows(torch.randn((24, c), device="cuda"))
    r = torch.tensor([0, 262143, 262144, n - 1], device="cuda")
    X, W = (block.q8_values(a.view(torch.uint8).cpu().numpy(), b.view(torch.uint8).cpu().numpy())
            for a, b in ((q.view(torch.uint8)[r], s.view(torch.uint8)[r]), wq))
    for out in (F32, BF16):
        Y = X @ W.T
        within(sp.sp_q8_linear((q, s), wq, out)[r], Y, q8_bound(X, W, Y, out), "z")
    del q, s
    torch.cuda.empty_cache()
