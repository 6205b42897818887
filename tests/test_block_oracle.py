"""Pins of oracle/block.py: against torch's autograd in float64, against differences, and against torch's own 8-bit type; and the
refusals of the block operators' C entry points, which need no GPU."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import block

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_13846_amd", "libsp_conv.so")


@pytest.mark.parametrize("split", [False, True])
def test_rope_is_a_turn_and_its_gradient_turns_back(split):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((5, 3, 14)), rng.standard_normal((5, 3, 14))
    pos = rng.integers(-40, 40, (5, 3))
    parts = (4, 0, 6)
    y = block.rope(x, pos, parts, split=split, scale=0.5)
    assert np.array_equal(y[:, :, 10:], x[:, :, 10:])                     # what no axis turns
    assert np.allclose((y ** 2).sum(2), (x ** 2).sum(2))                  # lengths stay
    z, at = x[:, :, :10], 0
    want = []
    for a, part in enumerate(parts):                                      # as complex numbers
        b = z[:, :, at:at + part]
        pair = b[..., :part // 2] + 1j * b[..., part // 2:] if split else b[..., ::2] + 1j * b[..., 1::2]
        turned = pair * np.exp(1j * (pos[:, a, None] * 0.5 * 10000.0 ** (-2 * np.arange(part // 2) / max(part, 1))))[:, None]
        want.append(np.concatenate([turned.real, turned.imag], 2) if split else np.stack([turned.real, turned.imag], 3).reshape(5, 3, part))
        at += part
    assert np.allclose(y[:, :, :10], np.concatenate(want, 2))
    dx = block.rope(dy, pos, parts, split=split, scale=0.5, back=True)
    assert abs((dx * x).sum() - (dy * y).sum()) < 1e-10                   # y is linear in x
    assert np.allclose(block.rope(y, pos, parts, split=split, scale=0.5, back=True), x)


def test_rms_matches_autograd():
    rng = np.random.default_rng(1)
    h, dy, dh, gamma = rng.standard_normal((9, 13)), rng.standard_normal((9, 13)), rng.standard_normal((9, 13)), rng.standard_normal(13)
    y, rstd = block.rms_fwd(h, gamma, 1e-3)
    t, tg = torch.tensor(h, requires_grad=True), torch.tensor(gamma, requires_grad=True)
    want = t * (t.square().mean(1, keepdim=True) + 1e-3).rsqrt() * tg
    assert np.allclose(y, want.detach().numpy())
    grads = torch.autograd.grad((want * torch.tensor(dy)).sum() + (t * torch.tensor(dh)).sum(), (t, tg))
    for got, ref in zip(block.rms_bwd(h, dy, gamma, rstd, dh), grads):
        assert np.allclose(got, ref.numpy())


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_ffn_matches_autograd_and_differences(act):
    rng = np.random.default_rng(4)
    x, w_in, w_out, dy = rng.standard_normal((6, 5)), rng.standard_normal((14, 5)), rng.standard_normal((5, 7)), rng.standard_normal((6, 5))
    y, g, u, h = block.ffn_fwd(x, w_in, w_out, act)
    t = [torch.tensor(a, requires_grad=True) for a in (x, w_in, w_out)]
    gu = t[0] @ t[1].T
    want = (getattr(torch.nn.functional, act)(gu[:, :7]) * gu[:, 7:]) @ t[2].T
    assert np.allclose(y, want.detach().numpy())
    grads = block.ffn_bwd(x, w_in, w_out, g, u, h, dy, act)[:3]
    for got, ref in zip(grads, torch.autograd.grad(want, t, torch.tensor(dy))):
        assert np.allclose(got, ref.numpy())
    for which, at in ((0, (2, 3)), (1, (3, 1)), (1, (10, 4)), (2, (4, 6))):
        both = []
        for sign in (1, -1):
            args = [a.copy() for a in (x, w_in, w_out)]
            args[which][at] += sign * 1e-6
            both.append((block.ffn_fwd(*args, act)[0] * dy).sum())
        assert abs((both[0] - both[1]) / 2e-6 - grads[which][at]) < 1e-6


def test_codes_are_those_of_the_type():
    v = torch.cat([torch.linspace(-448, 448, 5001), torch.randn(4000) * 0.02, torch.tensor([0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, 464.0 / 2])])
    want = v.to(torch.float8_e4m3fn)
    assert np.array_equal(block.e4m3_codes(v.double().numpy()), want.view(torch.uint8).numpy())
    every = np.arange(256, dtype=np.uint8)
    assert np.array_equal(block.e4m3(every), torch.tensor(every).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_scales_are_the_least():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 300)) * 2.0 ** rng.integers(-60, 60, (40, 1))
    x[3, :128], x[4, 5], x[5, 200], x[6, 0] = 0, np.inf, np.nan, 448.0
    x[7, :128] = 2.0 ** -140
    x[8, 0] = 448 * 2.0 ** 100
    codes, scales = block.q8_rows(x)
    assert codes.shape == (40, 384) and scales.shape == (40, 4) and (scales[:, 3] == 127).all()
    assert scales[3, 0] == 127 and scales[4, 0] == 255 and scales[5, 1] == 255 and scales[7, 0] == 0 and scales[8, 0] == 227
    back = block.q8_values(codes, scales)
    assert np.isnan(back[4, :128]).all() and np.isfinite(back[4, 128:]).all() and not codes[:, 300:].any()
    for r in (0, 1, 2, 6, 9, 20, 39):
        for b in range(3):
            top = np.abs(x[r, 128 * b:128 * b + 128]).max()
            unit = 2.0 ** (int(scales[r, b]) - 127)
            assert 224 * unit < top <= 448 * unit
        assert (np.abs(back[r, :300] - x[r]) <= np.maximum(np.abs(x[r]) / 16, np.repeat(2.0 ** (scales[r, :3].astype(float) - 127), 128)[:300] / 1024)).all()


# ---- refusals --------------------------------------------------------------------------------------------------
class Rope(C.Structure):
    _fields_ = [("n", C.c_int64), ("heads", C.c_int32), ("dim", C.c_int32), ("axes", C.c_int32), ("part", C.c_int32 * 4), ("split", C.c_int32),
                ("base", C.c_double), ("scale", C.c_double), ("dt", C.c_int32), ("d_pos", C.c_void_p), ("ld_pos", C.c_int64)]


class Ffn(C.Structure):
    _fields_ = [("n", C.c_int64), ("c", C.c_int32), ("m", C.c_int32), ("act", C.c_int32), ("dt", C.c_int32)]


@pytest.fixture(scope="module")
def lib():
    l = C.CDLL(LIB)
    l.sp_last_error.restype = C.c_char_p
    for name in ("sp_rms_norm_bwd_work", "sp_q8_codes_bytes", "sp_q8_scales_bytes", "sp_q8_linear_work", "sp_ffn_work_bytes"):
        getattr(l, name).restype = C.c_int64
    return l


INVALID, UNSUPPORTED = -1, -5
P = C.c_void_p(4096)   # never read: every call is refused, or has no rows


def i8(v):
    return C.c_int64(v)


def test_rope_refusals(lib):
    def call(ldx=12, ldy=12, x=P, y=P, **change):
        a = dict(n=3, heads=2, dim=6, axes=2, part=(C.c_int32 * 4)(2, 4), split=0, base=1e4, scale=1.0, dt=0, d_pos=4096, ld_pos=2)
        a.update(change)
        return lib.sp_rope_fwd(C.byref(Rope(**a)), x, i8(ldx), y, i8(ldy), None)

    assert call(n=0) == 0 and call(n=0, x=None, y=None, d_pos=None) == 0
    assert lib.sp_rope_fwd(None, P, i8(12), P, i8(12), None) == INVALID and lib.sp_rope_bwd(None, P, i8(12), P, i8(12), None) == INVALID
    for change in (dict(n=-1), dict(heads=0), dict(dim=0), dict(axes=0), dict(axes=5), dict(part=(C.c_int32 * 4)(3, 2)),
                   dict(part=(C.c_int32 * 4)(4, 4)), dict(part=(C.c_int32 * 4)(-2, 4)), dict(base=0.0), dict(base=float("nan")),
                   dict(base=float("inf")), dict(scale=float("inf")), dict(dt=2), dict(ld_pos=1), dict(ldx=11), dict(ldy=11), dict(d_pos=None),
                   dict(x=None), dict(y=None), dict(ldx=12, ldy=14), dict(part=(C.c_int32 * 4)(2 ** 31 - 2, 2 ** 31 - 2))):
        assert call(**change) == INVALID, change
        assert lib.sp_last_error()
    assert call(dim=258, ldx=516, ldy=516) == UNSUPPORTED


def test_rms_refusals(lib):
    f = C.c_float

    def fwd(x=P, res=P, n=3, c=8, gamma=P, eps=1e-5, h=C.c_void_p(8192), y=C.c_void_p(12288), rstd=P, dt=1):
        return lib.sp_rms_norm_fwd(x, res, i8(n), c, gamma, f(eps), h, y, rstd, dt, None)

    def q8(x=P, res=None, n=3, c=8, gamma=P, eps=1e-5, h=None, q=P, s=P, dt=1):
        return lib.sp_rms_norm_q8(x, res, i8(n), c, gamma, f(eps), h, q, s, dt, None)

    def bwd(h=P, dy=P, dh=None, n=3, c=8, gamma=P, rstd=P, dx=P, dgamma=P, work=P, dt=1):
        return lib.sp_rms_norm_bwd(h, dy, dh, i8(n), c, gamma, rstd, dx, dgamma, work, dt, None)

    assert fwd(n=0) == 0 and q8(n=0) == 0 and fwd(n=0, x=None, y=None, rstd=None) == 0
    for bad in (dict(n=-1), dict(c=0), dict(c=65537), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(gamma=None), dict(dt=3)):
        assert fwd(**bad) == INVALID and q8(**bad) == INVALID, bad
    for bad in (dict(y=None), dict(rstd=None), dict(h=None), dict(res=None), dict(y=C.c_void_p(8192))):
        assert fwd(**bad) == INVALID, bad
    for bad in (dict(q=None), dict(s=None), dict(res=P), dict(h=P), dict(q=C.c_void_p(4104))):
        assert q8(**bad) == INVALID, bad
    for bad in (dict(n=-1), dict(c=0), dict(c=65537), dict(h=None), dict(dy=None), dict(gamma=None), dict(rstd=None), dict(dx=None), dict(dgamma=None),
                dict(work=None), dict(dt=-1)):
        assert bwd(**bad) == INVALID, bad
    assert lib.sp_rms_norm_bwd_work(i8(-1), 8, 0) == -1 and lib.sp_rms_norm_bwd_work(i8(5), 0, 0) == -1
    assert lib.sp_rms_norm_bwd_work(i8(5), 8, 0) >= 32


def test_q8_refusals(lib):
    def rows(x=P, ldx=8, n=3, c=8, turned=0, q=P, s=P, dt=1):
        return lib.sp_q8_rows(x, i8(ldx), i8(n), c, turned, q, s, dt, None)

    def linear(q=P, s=P, n=3, c=8, wq=P, ws=P, m=4, y=P, dt=1, work=P):
        return lib.sp_q8_linear(q, s, i8(n), i8(c), wq, ws, i8(m), y, dt, work, None)

    assert rows(n=0) == 0 and linear(n=0) == 0
    for bad in (dict(n=-1), dict(c=0), dict(ldx=7), dict(x=None), dict(q=None), dict(s=None), dict(q=C.c_void_p(4100)), dict(dt=2)):
        assert rows(**bad) == INVALID, bad
    for bad in (dict(n=-1), dict(c=0), dict(m=0), dict(q=None), dict(s=None), dict(wq=None), dict(ws=None), dict(y=None), dict(work=None), dict(dt=7),
                dict(q=C.c_void_p(4104)), dict(wq=C.c_void_p(4104)), dict(s=C.c_void_p(4098)), dict(work=C.c_void_p(4112))):
        assert linear(**bad) == INVALID, bad
    assert linear(c=2 ** 22 + 1) == UNSUPPORTED and linear(n=2 ** 30 + 1) == UNSUPPORTED
    assert lib.sp_q8_codes_bytes(i8(3), i8(129)) == 768 and lib.sp_q8_scales_bytes(i8(3), i8(129)) == 12 and lib.sp_q8_scales_bytes(i8(3), i8(513)) == 24
    assert lib.sp_q8_codes_bytes(i8(-1), i8(1)) == -1 and lib.sp_q8_scales_bytes(i8(1), i8(0)) == -1 and lib.sp_q8_linear_work(i8(1), i8(0), i8(1)) == -1


def test_ffn_refusals(lib):
    def fwd(x=P, w=P, o=P, y=P, work=P, **change):
        a = dict(n=3, c=8, m=16, act=0, dt=1)
        a.update(change)
        return lib.sp_ffn_fwd(C.byref(Ffn(**a)), x, w, o, None, y, work, None)

    def bwd(x=P, w=P, o=P, kept=P, dy=P, dx=P, dw=P, do=P, work=P, **change):
        a = dict(n=3, c=8, m=16, act=0, dt=1)
        a.update(change)
        return lib.sp_ffn_bwd(C.byref(Ffn(**a)), x, w, o, kept, dy, dx, dw, do, work, None)

    assert fwd(n=0) == 0
    assert lib.sp_ffn_fwd(None, P, P, P, None, P, P, None) == INVALID
    for bad in (dict(n=-1), dict(c=0), dict(m=0), dict(act=2), dict(dt=2), dict(x=None), dict(w=None), dict(o=None), dict(work=None),
                dict(work=C.c_void_p(4112))):
        assert fwd(**bad) == INVALID and bwd(**bad) == INVALID, bad
    assert fwd(y=None) == INVALID
    for bad in (dict(kept=None), dict(dy=None), dict(dx=None), dict(dw=None), dict(do=None)):
        assert bwd(**bad) == INVALID, bad
    assert fwd(c=2 ** 18 + 1) == UNSUPPORTED and fwd(m=2 ** 18 + 1) == UNSUPPORTED and fwd(n=2 ** 30 + 1) == UNSUPPORTED
    assert lib.sp_ffn_work_bytes(C.byref(Ffn(3, 8, 16, 0, 1)), 0) >= 3 * 16 * 2 and lib.sp_ffn_work_bytes(C.byref(Ffn(3, 8, 0, 0, 1)), 1) == -1


def test_parts_of_a_head_are_whole_numbers_whatever_was_asked_before():
    from paper_2012_13846_amd import binding
    x, pos = torch.zeros((2, 1, 32)), torch.zeros((2, 3), dtype=torch.int32)
    for call in (binding.sp_rope_fwd, binding.sp_rope_bwd):
        with pytest.raises(ValueError, match="CUDA"):                     # these parts would do
            call(x, pos, (12, 10, 10))
        for bad in ((12.0, 10.0, 10.0), (12, 10, 10.0), ("12",)):
            with pytest.raises(TypeError):
                call(x, pos, bad)
        for bad in ((), (2, 2, 2, 2, 2), (34,), (-2,)):
            with pytest.raises(ValueError, match="axes"):
                call(x, pos, bad)


def test_products_of_more_results_than_a_launch_has_threads_for_are_refused(lib):
    linear = lambda n, m, dt: lib.sp_q8_linear(P, P, i8(n), i8(128), P, P, i8(m), P, dt, P, None)  # noqa: E731
    for n, m in ((2 ** 30, 2 ** 30), (2 ** 30, 2 ** 12), (2 ** 12, 2 ** 30)):
        assert lib.sp_q8_linear_work(i8(n), i8(128), i8(m)) == -1 and linear(n, m, 0) == UNSUPPORTED and linear(n, m, 1) == UNSUPPORTED
    for dt in (0, 1):
        f = C.byref(Ffn(2 ** 30, 64, 2 ** 18, 0, dt))
        assert lib.sp_ffn_work_bytes(f, 0) == -1 and lib.sp_ffn_work_bytes(f, 1) == -1
        assert lib.sp_ffn_fwd(f, P, P, P, None, P, P, None) == UNSUPPORTED
        assert lib.sp_ffn_bwd(f, P, P, P, P, P, P, P, P, P, None) == UNSUPPORTED
        f = C.byref(Ffn(2 ** 18, 2 ** 13, 2 ** 15, 0, dt))                # large, and taken
        assert lib.sp_ffn_work_bytes(f, 0) > 2 ** 34 and lib.sp_ffn_work_bytes(f, 1) > 2 ** 34
    assert lib.sp_q8_linear_work(i8(2 ** 18), i8(2 ** 15), i8(2 ** 18)) >= 256 and lib.sp_q8_linear_work(i8(2 ** 30), i8(128), i8(64)) >= 256


def test_sizes_in_8_bits_beyond_64_bits_are_refused(lib):
    far = 2 ** 40
    assert lib.sp_q8_codes_bytes(i8(far), i8(far)) == -1 and lib.sp_q8_codes_bytes(i8(2 ** 24), i8(far)) == -1
    assert lib.sp_q8_scales_bytes(i8(far), i8(far)) == -1
    assert lib.sp_q8_codes_bytes(i8(2 ** 22), i8(far)) == 2 ** 62 and lib.sp_q8_scales_bytes(i8(2 ** 22), i8(far)) == 2 ** 55
    assert lib.sp_q8_codes_bytes(i8(0), i8(far)) == 0
