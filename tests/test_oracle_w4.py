"""Pins of the oracle of 4-bit weights with a scale per group, and the argument checks of include/qc_w4.h.  CPU only."""
import ctypes as C

import numpy as np
import pytest

from oracle import quant as Q
from oracle import w4 as W4


@pytest.fixture(scope="module")
def qc():
    import paper_2503_02508_amd as m
    return m


def test_hand_example():
    w = np.array([[7.0, -3.5, 0.5, 1.5, -7.0] + [0.0] * 11, [0.0] * 16, [-1.0, 2.0, 14.0] + [0.0] * 13], np.float32)
    u, s, z = W4.group_quant(w, 32, False)
    assert s[:, 0].tolist() == [1.0, 1.0, 2.0] and (z == 8).all()
    assert u[0, :5].tolist() == [15, 4, 8, 10, 1] and (u[1] == 8).all()          # halves go to even
    assert u[2, :3].tolist() == [8, 9, 15]                                       # -0.5 -> 0, 1, 7
    u, s, z = W4.group_quant(w, 32, True)
    assert s[2, 0] == 1.0 and z[2, 0] == 1 and u[2, :4].tolist() == [0, 3, 15, 1]
    assert s[1, 0] == 1.0 and z[1, 0] == 0 and (u[1] == 0).all()


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("N,K,group", [(5, 16, 32), (7, 144, 64), (3, 272, 128)])
def test_half_a_step_and_exact_zero(N, K, group, asym):
    rng = np.random.default_rng(K)
    w = (rng.standard_normal((N, K)) * rng.uniform(1e-4, 2, (N, 1)) + 0.3).astype(np.float32)
    w[:, ::7] = 0
    u, s, z = W4.group_quant(w, group, asym)
    v = W4.values(u, s, z, group)
    step = np.repeat(s, group, 1)[:, :K]
    # a zero point rounded by half a step moves one end of the range by half a step
    assert (np.abs(v - w) <= step * (1.001 if asym else 0.5001)).all()
    assert (v[w == 0] == 0).all()
    assert np.array_equal(W4.unpack(W4.pack(u)), u)


def test_one_group_is_the_row_quantiser():
    w = (np.random.default_rng(1).standard_normal((9, 128)) * 0.02).astype(np.float32)
    u, s, _ = W4.group_quant(w, 128, False)
    q, sw, _ = Q.weight_quant(w, 4)
    assert np.array_equal(u - 8, q) and np.array_equal(s[:, 0], sw)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_activation_derivative_and_gradients_against_differences(name):
    v = np.linspace(-9, 9, 181)
    h = 1e-5
    assert np.allclose((W4.act(name, v + h)[0] - W4.act(name, v - h)[0]) / (2 * h), W4.act(name, v)[1], atol=1e-9)
    rng = np.random.default_rng(2)
    x, Wg, Wu = rng.standard_normal((3, 16)), rng.standard_normal((5, 16)), rng.standard_normal((5, 16))
    bg, bu, dh = rng.standard_normal(5), rng.standard_normal(5), rng.standard_normal((3, 5))
    dg, du = W4.gated_grad(x, Wg, Wu, bg, bu, name, dh)
    dx = dg @ Wg + du @ Wu
    num = np.empty_like(x)
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = h
        num[i] = ((W4.gated(x + e, Wg, Wu, bg, bu, name) - W4.gated(x - e, Wg, Wu, bg, bu, name)) * dh).sum() / (2 * h)
    assert np.allclose(num, dx, atol=1e-7)


# ---------------------------------------------------------------- refusals, before any device call
P = 0x10000


def _desc(qc, N=8, K=64, group=32, q=P, scale=P, zero=None, sum=P):  # noqa: A002
    from paper_2503_02508_amd.binding import W4WeightDesc
    return W4WeightDesc(q, scale, zero, sum, N, K, group)


BAD_WEIGHTS = [(dict(q=None), -1), (dict(scale=None), -1), (dict(N=-1), -2), (dict(K=0), -2), (dict(K=24), -2), (dict(K=-16), -2),
               (dict(N=1 << 22), -2), (dict(K=1 << 22), -2), (dict(group=0), -7), (dict(group=16), -7), (dict(group=96), -7), (dict(group=-32), -7),
               (dict(N=(1 << 22) - 1, K=1 << 15), -7), (dict(q=P + 8), -3), (dict(scale=P + 2), -3), (dict(sum=P + 1), -3)]


@pytest.mark.parametrize("kw,code", BAD_WEIGHTS)
def test_every_call_refuses_a_bad_weight(qc, kw, code):
    L, bad, ok = qc.lib, C.byref(_desc(qc, **kw)), C.byref(_desc(qc))
    far = (1 << 22) - 16
    assert L.qc_w4_quantize(P, 0, far, bad, None) == code and qc.last_error()
    assert L.qc_w4_expand(bad, P, 0, far, None) == code
    assert L.qc_w4_linear(P, 0, far, 1.0, 128, bad, None, 1, P, far, None) == code
    assert L.qc_w4_gated(P, 0, far, 1.0, 128, bad, ok, None, None, 0, 1, P, far, None) == code
    assert L.qc_w4_gated(P, 0, far, 1.0, 128, ok, bad, None, None, 0, 1, P, far, None) == code
    assert L.qc_w4_linear_grad(P, 0, far, bad, None, 0, None, 1, P, far, None) == code
    assert L.qc_w4_linear_grad(P, 0, far, ok, P, far, bad, 1, P, far, None) == code
    assert L.qc_w4_gated_grad(P, 0, far, bad, ok, None, None, 0, P, far, 1, P, P, far, None) == code
    assert L.qc_w4_gated_grad(P, 0, far, ok, bad, None, None, 0, P, far, 1, P, P, far, None) == code


def test_refusals_of_the_other_arguments(qc):
    L, w = qc.lib, C.byref(_desc(qc))                                    # 8 x 64
    nosum, zeros, wide, short = (C.byref(_desc(qc, **kw)) for kw in (dict(sum=None), dict(zero=P), dict(K=128), dict(N=7)))
    for args, code in [((P, 3, 64, w, None), -7), ((P, 4, 64, w, None), -7), ((P, -1, 64, w, None), -7), ((None, 0, 64, w, None), -1),
                       ((P, 0, 63, w, None), -2), ((P, 0, 66, w, None), -3), ((P + 4, 0, 64, w, None), -3), ((P, 1, 68, w, None), -3),
                       ((P, 0, 1 << 22, w, None), -2), ((P, 0, 64, None, None), -1)]:
        assert L.qc_w4_quantize(*args) == code, args
    for args, code in [((w, P, 3, 64, None), -7), ((w, None, 0, 64, None), -1), ((w, P, 0, 60, None), -2), ((w, P + 2, 0, 64, None), -3),
                       ((w, P + 1, 2, 64, None), -3), ((None, P, 0, 64, None), -1)]:
        assert L.qc_w4_expand(*args) == code, args

    def linear(x=P, t=0, ldx=64, xs=1.0, zp=128, w=w, b=None, M=4, y=P, ldy=8):
        return L.qc_w4_linear(x, t, ldx, xs, zp, w, b, M, y, ldy, None)
    for kw, code in [(dict(x=None), -1), (dict(y=None), -1), (dict(t=5), -7), (dict(t=-1), -7), (dict(ldx=60), -2), (dict(ldy=7), -2),
                     (dict(x=P + 8), -3), (dict(ldx=66), -3), (dict(t=1, ldx=68), -3), (dict(t=3, ldx=72), -3), (dict(y=P + 2), -3), (dict(b=P + 2), -3),
                     (dict(M=-1), -2), (dict(M=1 << 24), -2), (dict(t=3, xs=0.0), -4), (dict(t=3, xs=float("nan")), -4),
                     (dict(t=3, xs=float("inf")), -4), (dict(t=3, zp=256), -4), (dict(t=3, zp=-1), -4), (dict(t=3, w=nosum), -1),
                     (dict(M=(1 << 24) - 1, w=C.byref(_desc(qc, N=256)), ldy=256), -7)]:
        assert linear(**kw) == code, kw
    assert linear(M=0) == 0 and linear(M=0, x=None, y=None) == 0
    assert linear(w=C.byref(_desc(qc, N=0, q=None, scale=None, sum=None)), y=None) == 0

    def gated(g=w, u=w, act=0, t=0, x=P, ldx=64, h=P, ldh=8, M=4, bg=None, bu=None, xs=1.0, zp=0):
        return L.qc_w4_gated(x, t, ldx, xs, zp, g, u, bg, bu, act, M, h, ldh, None)
    for kw, code in [(dict(u=wide), -2), (dict(u=short), -2), (dict(u=C.byref(_desc(qc, group=64))), -2), (dict(u=zeros), -7), (dict(g=zeros), -7),
                     (dict(act=2), -7), (dict(act=-1), -7), (dict(t=4), -7), (dict(x=None), -1), (dict(h=None), -1), (dict(h=P + 2), -3),
                     (dict(ldh=7), -2), (dict(bg=P + 1), -3), (dict(bu=P + 1), -3), (dict(t=3, u=nosum), -1), (dict(t=3, g=nosum), -1),
                     (dict(t=3, zp=300), -4), (dict(M=-2), -2)]:
        assert gated(**kw) == code, kw
    assert gated(M=0) == 0

    def lgrad(dy=P, t=0, ld=8, w=w, dy2=None, ld2=0, w2=None, M=4, dx=P, lddx=64):
        return L.qc_w4_linear_grad(dy, t, ld, w, dy2, ld2, w2, M, dx, lddx, None)
    for kw, code in [(dict(dy=None), -1), (dict(dx=None), -1), (dict(t=3), -7), (dict(ld=7), -2), (dict(lddx=63), -2), (dict(dy=P + 2), -3),
                     (dict(dx=P + 2), -3), (dict(t=1, dx=P + 1), -3), (dict(w2=w, ld2=8), -1), (dict(w2=w, dy2=P, ld2=7), -2),
                     (dict(w2=wide, dy2=P, ld2=8), -2), (dict(w2=zeros, dy2=P, ld2=8), -7), (dict(M=-1), -2), (dict(M=1 << 24), -2)]:
        assert lgrad(**kw) == code, kw
    assert lgrad(M=0) == 0 and lgrad(M=0, dy=None, dx=None) == 0

    def ggrad(g=w, u=w, act=0, t=0, x=P, ldx=64, dh=P, lddh=8, M=4, dg=P, du=P, ldd=8, bg=None, bu=None):
        return L.qc_w4_gated_grad(x, t, ldx, g, u, bg, bu, act, dh, lddh, M, dg, du, ldd, None)
    for kw, code in [(dict(t=3), -7), (dict(u=short), -2), (dict(u=zeros), -7), (dict(act=3), -7), (dict(x=None), -1), (dict(dh=None), -1),
                     (dict(dg=None), -1), (dict(du=None), -1), (dict(lddh=7), -2), (dict(ldd=7), -2), (dict(dh=P + 1), -3), (dict(dg=P + 2), -3),
                     (dict(du=P + 3), -3), (dict(bg=P + 1), -3), (dict(bu=P + 2), -3), (dict(M=-1), -2)]:
        assert ggrad(**kw) == code, kw
    assert ggrad(M=0) == 0


def test_the_binding_refuses_what_the_c_abi_cannot_see(qc):
    import torch
    ok = dict(N=4, K=64, group=32, device="cpu")
    w = qc.W4Weight.empty(**ok)
    assert (w.N, w.K, w.group) == (4, 64, 32) and w.zero is None and qc.W4Weight.empty(asymmetric=True, **ok).zero.shape == (4, 2)
    for bad in (dict(q=w.q.to(torch.int8)), dict(scale=w.scale.double()), dict(scale=w.scale[:, :1]), dict(zero=torch.zeros(4, 2)),
                dict(zero=torch.zeros(4, 3, dtype=torch.uint8)), dict(sum=torch.zeros(5)), dict(scale=torch.zeros(2, 4).t()),
                dict(q=torch.zeros((4, 64), dtype=torch.uint8)[:, ::2]), dict(group=64)):
        with pytest.raises(qc.QCError):
            qc.W4Weight(**{**dict(q=w.q, scale=w.scale, group=32, zero=w.zero, sum=w.sum), **bad})
    x, y = torch.zeros(2, 64), torch.zeros(2, 4)
    for args, kw in [((x.double(), w, y), {}), ((x[:, :48], w, y), {}), ((x, w, y[:1]), {}), ((x, w, y.half()), {}), ((x, w, y, torch.zeros(5)), {}),
                     ((x, w, y, torch.zeros(4).half()), {}), ((torch.zeros(64, 2).t(), w, y), {}), ((x.view(2, 8, 8), w, y), {}),
                     ((x.to(torch.int8), w, y.half()), {}), ((x, w, y), {})]:               # the last: not on a GPU
        with pytest.raises(qc.QCError):
            qc.qc_w4_linear(*args, **kw)
    with pytest.raises(qc.QCError):
        qc.qc_w4_linear_grad(y, w, x, dy2=y)
    with pytest.raises(qc.QCError):
        qc.qc_w4_gated_grad(x, w, w, y, y, torch.zeros(2, 8)[:, :4])


def test_weights_without_rows_may_lie_nowhere(qc):
    """N = 0 does nothing, also where the sums of 8-bit inputs or the zero points of a pair have no memory."""
    L, none = qc.lib, C.byref(_desc(qc, N=0, q=None, scale=None, sum=None))
    zeros = C.byref(_desc(qc, zero=P))
    assert L.qc_w4_linear(P, 3, 64, 0.02, 100, none, None, 4, None, 0, None) == 0
    assert L.qc_w4_gated(P, 3, 64, 0.02, 100, none, none, None, None, 0, 4, None, 0, None) == 0
    assert L.qc_w4_gated(P, 3, 64, 0.02, 100, none, C.byref(_desc(qc, N=0, zero=P)), None, None, 0, 4, None, 0, None) == 0
    for a, b in ((none, zeros), (zeros, none)):
        assert L.qc_w4_linear_grad(P, 0, 8, a, P, 8, b, 0, P, 64, None) == 0


def test_gradients_of_results_may_be_larger_than_results(qc):
    """The limit of 2^31 elements is the result's, dx; the arguments are checked up to the missing dx."""
    L, w = qc.lib, C.byref(_desc(qc, N=1 << 18, K=16))
    assert L.qc_w4_linear_grad(P, 2, 1 << 18, w, None, 0, None, 1 << 14, None, 16, None) == -1
    assert L.qc_w4_linear_grad(P, 2, 1 << 18, w, P, 1 << 18, w, 1 << 14, None, 16, None) == -1
    assert L.qc_w4_linear_grad(P, 2, 8, C.byref(_desc(qc, K=1 << 18)), None, 0, None, 1 << 14, P, 1 << 18, None) == -7


def test_tensors_of_other_dimensions_are_refused_like_other_shapes(qc):
    import torch
    w = qc.W4Weight.empty(4, 64, 32, device="cpu")
    for kw in (dict(group=0), dict(group=-32), dict(K=17), dict(K=0), dict(N=-1)):
        with pytest.raises(qc.QCError):
            qc.W4Weight.empty(**{**dict(N=4, K=64, group=32, device="cpu"), **kw})
    for q in (torch.zeros(32, dtype=torch.uint8), torch.zeros((), dtype=torch.uint8), torch.zeros((4, 4, 8), dtype=torch.uint8)):
        with pytest.raises(qc.QCError):
            qc.W4Weight(q, w.scale, 32)
    x, one = torch.zeros(2, 64), torch.zeros(())
    for call, args in ((qc.qc_w4_linear, (one, w, x)), (qc.qc_w4_gated, (one, w, w, x)), (qc.qc_w4_linear_grad, (one, w, x)),
                       (qc.qc_w4_gated_grad, (one, w, w, x, x, x)), (qc.qc_w4_quantize, (one, w)), (qc.qc_w4_expand, (w, one))):
        with pytest.raises(qc.QCError):
            call(*args)
