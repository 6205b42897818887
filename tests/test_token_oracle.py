"""Pins of oracle/tokens.py: against torch's autograd in float64 and against differences of the forward pass; and the
refusals of the token operators' C entry points, which need no GPU."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import tokens

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_13846_amd", "libsp_conv.so")


def test_layer_norm_matches_autograd():
    rng = np.random.default_rng(1)
    x, dy, gamma, beta = rng.standard_normal((9, 13)), rng.standard_normal((9, 13)), rng.standard_normal(13), rng.standard_normal(13)
    y, mean, rstd = tokens.layer_norm_fwd(x, gamma, beta, 1e-5)
    t = [torch.tensor(a, requires_grad=True) for a in (x, gamma, beta)]
    want = torch.nn.functional.layer_norm(t[0], (13,), t[1], t[2], 1e-5)
    assert np.allclose(y, want.detach().numpy(), rtol=1e-12, atol=1e-12)
    for got, ref in zip(tokens.layer_norm_bwd(x, dy, gamma, mean, rstd), torch.autograd.grad(want, t, torch.tensor(dy))):
        assert np.allclose(got, ref.numpy(), rtol=1e-10, atol=1e-11)


@pytest.mark.parametrize("a,b,left,right,sinks", [(7, 7, 2, 0, 1), (5, 9, 3, 1, 2), (6, 3, 1, 0, 0), (4, 4, 9, 9, 0), (3, 0, 2, 0, 1)])
def test_window_attention_matches_autograd_and_differences(a, b, left, right, sinks):
    rng = np.random.default_rng(a * 10 + b)
    h, kv, d = 4, 2, 3
    q, k, v, do = rng.standard_normal((a, h, d)), rng.standard_normal((b, kv, d)), rng.standard_normal((b, kv, d)), rng.standard_normal((a, h, d))
    qs, ks = [0, a], [0, b]
    o, lse, _ = tokens.window_attn_fwd(q, k, v, qs, ks, left, right, sinks, 0.7)
    (dq, dk, dv), _ = tokens.window_attn_bwd(q, k, v, o, do, lse, qs, ks, left, right, sinks, 0.7)
    t = [torch.tensor(x, requires_grad=True) for x in (q, k, v)]
    seen = torch.zeros((a, b), dtype=torch.bool)
    for i in range(a):                                     # the rule, pair by pair
        for j in range(b):
            p = i + b - a
            seen[i, j] = j <= p + right and (p - left <= j or j < sinks)
    s = torch.einsum("ihd,jhd->hij", t[0], t[1].repeat_interleave(h // kv, 1)) * 0.7
    s = s.masked_fill(~seen, -torch.inf)
    some = seen.any(1)
    p = torch.where(some[:, None], torch.softmax(s.masked_fill(~some[:, None], 0.0), 2) if b else s, 0.0)
    want = torch.einsum("hij,jhd->ihd", p, t[2].repeat_interleave(h // kv, 1))
    assert np.allclose(o, want.detach().numpy(), atol=1e-12)
    assert np.array_equal(np.isneginf(lse), ~np.broadcast_to(some.numpy()[:, None], (a, h)))
    for got, ref in zip((dq, dk, dv), torch.autograd.grad(want, t, torch.tensor(do), allow_unused=True)):
        assert np.allclose(got, np.zeros_like(got) if ref is None else ref.numpy(), atol=1e-11)
    if b:
        at, step = (b - 1, 1, 2), 1e-6
        both = []
        for sign in (1, -1):
            k2 = k.copy()
            k2[at] += sign * step
            both.append((tokens.window_attn_fwd(q, k2, v, qs, ks, left, right, sinks, 0.7)[0] * do).sum())
        assert abs((both[0] - both[1]) / (2 * step) - dk[at]) < 1e-7


def test_keys_that_are_not_seen_do_not_reach_the_results():
    rng = np.random.default_rng(3)
    q, k, v, do = (rng.standard_normal((6, 1, 2)) for _ in range(4))
    o, lse, _ = tokens.window_attn_fwd(q, k, v, [0, 6], [0, 6], 1, 0, 0, 1.0)
    k2, v2 = k.copy(), v.copy()
    k2[1], v2[1] = np.nan, np.inf
    o2, lse2, _ = tokens.window_attn_fwd(q, k2, v2, [0, 6], [0, 6], 1, 0, 0, 1.0)
    assert np.array_equal(o[[0, 3, 4, 5]], o2[[0, 3, 4, 5]]) and np.array_equal(lse[3:], lse2[3:])
    assert not np.isfinite(o2[1:3]).any()


@pytest.mark.parametrize("left,sinks,cap", [(3, 2, 6), (3, 2, 40), (2, 0, 3), (50, 1, 8)])
def test_steps_through_the_ring_match_the_whole_sequence(left, sinks, cap):
    rng = np.random.default_rng(cap)
    n, h, kv, d = 23, 2, 1, 3
    q, k, v = rng.standard_normal((n, h, d)), rng.standard_normal((n, kv, d)), rng.standard_normal((n, kv, d))
    kc, vc = np.full((1, cap, kv, d), np.nan), np.full((1, cap, kv, d), np.nan)
    reach = min(left, cap - sinks - 1)                     # what a full ring still holds
    want, _, _ = tokens.window_attn_fwd(q, k, v, [0, n], [0, n], reach, 0, sinks, 0.6)
    for t in range(n):
        got, _ = tokens.window_attn_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], kc, vc, [t], left, sinks, 0.6)
        assert np.allclose(got[0], want[t], atol=1e-13)


def test_distillation_matches_autograd_and_differences():
    rng = np.random.default_rng(5)
    n, m, k, T = 6, 11, 4, 1.7
    z, top, w = rng.standard_normal((n, m)), rng.standard_normal((n, k)), rng.random(n)
    index = np.stack([rng.permutation(m)[:k] for _ in range(n)]).astype(np.int32)
    index[1, 2], index[2, :], index[3, 0] = -1, m, index[3, 1]          # padding, no entries, one column twice
    loss, dz = tokens.distill(z, top, index, T, w)
    t = torch.tensor(z, requires_grad=True)
    total = 0
    for r in range(n):
        ok = [j for j in range(k) if 0 <= index[r, j] < m]
        if ok:
            a = torch.softmax(torch.tensor(top[r, ok]) / T, 0)
            total = total + w[r] * T * T * (a * (a.log() - torch.log_softmax(t[r] / T, 0)[torch.tensor(index[r, ok]).long()])).sum()
    assert abs(loss - total.item()) < 1e-12
    assert np.allclose(dz, torch.autograd.grad(total, t)[0].numpy(), atol=1e-13)
    assert not dz[2].any()


def test_refusals_need_no_gpu():
    lib = ctypes.CDLL(LIB)
    lib.sp_last_error.restype = ctypes.c_char_p
    from paper_2012_13846_amd.binding import _WindowAttn
    i8, f = ctypes.c_int64, ctypes.c_float
    x = ctypes.c_void_p(4096)                              # never read: every call is refused before a launch
    assert lib.sp_layer_norm_fwd(x, i8(4), 0, x, x, f(1e-5), x, x, x, 0, None) == -1
    assert lib.sp_layer_norm_fwd(x, i8(-1), 8, x, x, f(1e-5), x, x, x, 0, None) == -1
    assert lib.sp_layer_norm_fwd(x, i8(4), 65537, x, x, f(1e-5), x, x, x, 0, None) == -1
    assert lib.sp_layer_norm_fwd(x, i8(4), 8, x, x, f(-1.0), x, x, x, 0, None) == -1
    assert lib.sp_layer_norm_fwd(x, i8(4), 8, x, x, f(float("nan")), x, x, x, 0, None) == -1
    assert lib.sp_layer_norm_fwd(x, i8(4), 8, x, x, f(1e-5), x, x, x, 2, None) == -1
    assert lib.sp_layer_norm_fwd(None, i8(4), 8, x, x, f(1e-5), x, x, x, 0, None) == -1
    assert lib.sp_layer_norm_fwd(None, i8(0), 8, x, x, f(1e-5), None, None, None, 0, None) == 0
    assert lib.sp_layer_norm_bwd(x, None, i8(4), 8, x, x, x, x, x, x, 0, None) == -1
    assert b"NULL" in lib.sp_last_error()

    def fwd(ld=64, q=x, **change):
        a = dict(n_q=4, n_k=4, n_clouds=1, heads=4, kv_heads=2, dim=16, left=3, right=0, sinks=0, scale=0.25, dt=1,
                 d_q_starts=4096, d_k_starts=4096)
        a.update(change)
        return lib.sp_window_attn_fwd(ctypes.byref(_WindowAttn(**a)), q, i8(ld), x, i8(ld), x, i8(ld), x, i8(ld), x, None)

    assert fwd(kv_heads=3) == -1 and fwd(heads=0) == -1 and fwd(dim=0) == -1 and fwd(n_q=-1) == -1 and fwd(n_clouds=-1) == -1
    assert fwd(left=-1) == -1 and fwd(right=-1) == -1 and fwd(sinks=-1) == -1 and fwd(scale=float("inf")) == -1 and fwd(dt=2) == -1
    assert fwd(scale=float("nan")) == -1 and fwd(d_q_starts=None) == -1 and fwd(q=None) == -1 and fwd(ld=63) == -1
    assert b"overlap" in lib.sp_last_error()
    assert fwd(dim=129, ld=4096) == -5 and fwd(n_k=2 ** 30 + 1) == -5 and fwd(ld=2 ** 33) == -5
    assert lib.sp_window_attn_fwd(None, x, i8(64), x, i8(64), x, i8(64), x, i8(64), x, None) == -1

    def step(batch=2, cap=8, heads=4, kv=2, dim=16, left=3, sinks=1, scale=0.25, dt=1, lens=x):
        return lib.sp_window_attn_step(x, x, x, x, x, lens, batch, cap, heads, kv, dim, left, sinks, f(scale), x, dt, None)

    assert step(batch=-1) == -1 and step(cap=1) == -1 and step(kv=3) == -1 and step(dim=0) == -1 and step(left=-1) == -1
    assert step(sinks=-1) == -1 and step(scale=float("nan")) == -1 and step(dt=3) == -1 and step(lens=None) == -1
    assert step(dim=200) == -5 and step(batch=0, lens=None) == 0

    def distill(n=2, m=8, k=2, temp=1.0, loss=x, dt=0, z=x):
        return lib.sp_distill(z, i8(n), m, x, x, k, f(temp), None, loss, x, dt, None)

    assert distill(n=-1) == -1 and distill(m=0) == -1 and distill(k=0) == -1 and distill(k=257) == -1 and distill(temp=0.0) == -1
    assert distill(temp=float("nan")) == -1 and distill(temp=float("inf")) == -1 and distill(loss=None) == -1 and distill(dt=5) == -1
    assert distill(z=None) == -1


def test_a_temperature_without_an_fp32_reciprocal_is_refused():
    lib = ctypes.CDLL(LIB)
    x = ctypes.c_void_p(4096)                              # never read
    for temp in (1e-38, 1e-40, -1e-30, 3.2e38):
        assert lib.sp_distill(x, ctypes.c_int64(2), 8, x, x, 2, ctypes.c_float(temp), None, x, x, 0, None) == -1


def test_a_window_wider_than_an_int32_is_no_narrow_one():
    from paper_2012_13846_amd.binding import _reach
    assert [_reach(v) for v in (0, 5, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 7, 2 ** 63)] == [0, 5] + [2 ** 31 - 1] * 5
    assert [_reach(v) for v in (-1, -2 ** 31, -2 ** 32, -2 ** 32 + 9)] == [-1] * 4   # refused by the library
