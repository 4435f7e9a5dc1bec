"""8-bit layers with a scale for each token (include/qc_t8.h) against the float64 oracle.

Codes, scales, sums with the residual and normalised rows are decided by the definition: equal bit for bit.  Tolerances of the rest, derived
from the arithmetic (e = 2^-24, half a float32 step; h = half a step of the result's type, absolute below its normal numbers):
  norm_grad  dx: four roundings of each of its terms, and rho^3 sum(g h) / K off by 4 e of itself and by 33 e sum |g h| (at most 32 terms one
             after the other, each of a rounded product)
             dweight: two roundings of each term, float32 sums of a group's rows (n of them), float64 sums of the groups
  gated_grad the logistic function to 9 e, value and derivative to 16 e of their terms; below 2^-126 both are subnormal float32 numbers, off
             by 2^-149 before the gradient multiplies them
  linear     the sum's conversion, two products and the addition: 4 e (|sum x_s w_s| + |bias|)
  linear_grad a term of dy w_s off by 1.01 * 2^-16 (2^-32) of the row's largest and by 4 e of itself, times |q|; the planes' sum and the last
             product by 4 e of their terms"""
import numpy as np
import pytest

from oracle import t8 as O

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
HALF = {"f32": E, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}
EPS = float(np.float32(1e-6))
TYPES = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def qc():
    import paper_2503_02508_amd as m
    return m


def _type(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _np(t):
    return t.double().cpu().numpy()


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _rows(rows, cols, dtype, pad=0, offset=0, fill=None):
    """[rows, cols] inside a larger buffer of known contents, and that buffer."""
    import torch
    buf = torch.full((rows + 2, cols + pad), 77, dtype=dtype, device="cuda")
    t = buf[1:1 + rows, offset:offset + cols]
    if fill is not None:
        t.copy_(fill)
    return t, buf


def _untouched(t, buf):
    b = buf.clone()
    r, c = t.shape
    o = (t.data_ptr() - buf.data_ptr()) // t.element_size() - buf.stride(0)
    b[1:1 + r, o:o + c] = 77
    return bool((b == 77).all())


def _check(got, want, tol, t, what):
    got = _np(got)
    lim = tol + HALF[t] * (np.abs(want) + tol) + TINY[t]
    bad = ~(np.abs(got - want) <= lim)
    assert not bad.any(), "%s: %d of %d, worst %g of its limit at %s" % (
        what, bad.sum(), bad.size, np.nanmax(np.abs(got - want) / lim), np.argwhere(bad)[:3].tolist())


def _same_codes(q, scale, v, what):
    want, s = O.codes(v)
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True), what
    got = q.cpu().numpy().astype(np.int64)
    assert np.array_equal(got, want), "%s: %d of %d codes" % (what, (got != want).sum(), want.size)


# rows, width: one element, one row, odd everything, a vector and a bit, several rows a wavefront, wide rows, rows that are read again
SHAPES = [(1, 1), (1, 8192), (3, 7), (40, 3), (6, 8), (7, 9), (5, 64), (2, 1153), (77, 1152), (9, 3081), (515, 40), (130, 513), (6000, 72), (17000, 33), (1500, 1153), (2100, 700), (1030, 4608), (2000, 9001), (3, 16384),
          (2, 16390), (1, 40000), (2, 131071)]


def _tokens(rng, M, K, t):
    x = rng.standard_normal((M, K)) * np.exp(rng.uniform(-3, 3, (M, 1)))
    x[:, rng.integers(0, K)] *= 8
    if M > 2:
        x[M // 2] = 0
    return _dev(x).to(_type(t))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,K", SHAPES)
def test_quantize_and_expand(qc, M, K, t):
    import torch
    rng = np.random.default_rng(M * 7 + K)
    for pad, off, qpad in ((0, 0, 0), (5, 3, 3), (16, 8, 16)):
        x, _ = _rows(M, K, _type(t), pad, off, _tokens(rng, M, K, t))
        q, qbuf = _rows(M, K, torch.int8, qpad)
        s = torch.empty(M, device="cuda")
        qc.qc_t8_quantize(x, q, s)
        _same_codes(q, s, _np(x).astype(np.float32), "%s pad %d" % (t, pad))
        assert _untouched(q, qbuf)
        for o in TYPES:
            out, buf = _rows(M, K, _type(o), qpad)
            qc.qc_t8_expand(q, s, out)
            want = (q.float() * s[:, None]).to(_type(o))
            assert torch.equal(out, want) and _untouched(out, buf)


@pytest.mark.parametrize("t", TYPES)
def test_quantize_borders(qc, t):
    """Quotients at and next to halves, a row whose largest value is its only one, equal values, signs."""
    import torch
    K = 512
    v = np.zeros((6, K), np.float64)
    v[0] = (np.arange(K) - 256) / 2.0
    v[0, 0] = 127
    v[1, 3] = -2.5
    v[2] = 1.0
    v[3] = np.where(np.arange(K) % 2, 0.75, -0.75)
    n = np.arange(K) % 253 / 2.0
    v[4] = np.nextafter(n.astype(np.float32), np.float32(0))
    v[4, 0] = 127
    v[5] = np.nextafter(n.astype(np.float32), np.float32(1e9))
    v[5, 0] = 127
    x = _dev(v).to(_type(t))
    for scale in (1.0, 0.37, 3e4 if t != "f16" else 3.0):
        xs = (x.double() * scale).to(_type(t))
        q, s = torch.empty((6, K), dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
        qc.qc_t8_quantize(xs, q, s)
        _same_codes(q, s, _np(xs).astype(np.float32), "%s scale %g" % (t, scale))


def test_quantize_extreme_rows(qc):
    """Rows of subnormal numbers, at the top of float32, with infinities and NaN: the others are not touched by them."""
    import torch
    v = np.random.default_rng(3).standard_normal((9, 100)).astype(np.float32)
    tiny = np.float32(2.0 ** -149)
    v[0] = 0
    v[0, :3] = [tiny, -tiny, 0]
    v[1] = tiny * np.arange(100, dtype=np.float32) * 2
    v[2] *= np.float32(1e-40)
    v[3] *= np.float32(3.0e38 / np.abs(v[3]).max())
    v[4, 5] = np.inf
    v[5, 99] = -np.inf
    v[6, 50] = np.nan
    v[7] *= np.float32(1e-30)
    for kern in (100, 99):
        x = _dev(v[:, :kern])
        q, s = torch.full((9, kern), 55, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
        qc.qc_t8_quantize(x, q, s)
        _same_codes(q, s, v[:, :kern], "extreme")
        out = torch.empty((9, kern), device="cuda")
        qc.qc_t8_expand(q, s, out)
        bad = ~torch.isfinite(x).all(1)
        assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,K", [s for s in SHAPES if s[0] * s[1] < 6e6])
def test_quantize_gated(qc, M, K, t, act):
    import torch
    rng = np.random.default_rng(M + K)
    x, _ = _rows(M, K, _type(t), 3, 1, _tokens(rng, M, K, t))
    g, _ = _rows(M, K, _type(t), 9, 4, _dev(rng.standard_normal((M, K)) * np.exp(rng.uniform(-2, 2, (M, 1)))).to(_type(t)))
    q, qbuf = _rows(M, K, torch.int8, 5)
    s = torch.empty(M, device="cuda")
    qc.qc_t8_quantize(x, q, s, gate=g, act=qc.QC_ACT_SILU if act == "silu" else qc.QC_ACT_GELU)
    # the oracle's own exponentials and sums are off by some 1e-15 of a value: where a quotient is that near to a border, and
    # nowhere else, its code may be either; none is at these seeds
    _same_codes(q, s, O.gated(_np(x), _np(g), act), "%s %s" % (t, act))
    assert _untouched(q, qbuf)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_quantize_gated_extremes(qc, act):
    """Gates far below zero (products that are subnormal, or nothing), far above, infinite; rows of zeros; large factors that bring small
    products back."""
    import torch
    rng = np.random.default_rng(5)
    K = 300
    x, g = rng.standard_normal((10, K)).astype(np.float32), rng.standard_normal((10, K)).astype(np.float32)
    g[0] = -np.abs(g[0]) * 40 - 60 if act == "silu" else -np.abs(g[0]) - 5
    x[0] = np.float32(1e30) * x[0]
    g[1] = 1e14
    x[1] *= np.float32(1e10)
    x[2] = 0
    g[3] = 0
    x[4, 7] = np.inf
    g[5, 8] = -np.inf
    g[6, 9] = np.inf
    g[7, 10] = np.nan
    g[8] = -1e9
    x[9] *= np.float32(1e-25)
    q, s = torch.full((10, K), 55, dtype=torch.int8, device="cuda"), torch.empty(10, device="cuda")
    qc.qc_t8_quantize(_dev(x), q, s, gate=_dev(g), act=qc.QC_ACT_SILU if act == "silu" else qc.QC_ACT_GELU)
    v = O.gated(x, g, act)
    if act == "silu":                   # the oracle's form loses an infinite gate
        v[5, 8] = v[6, 9] = np.nan
    _same_codes(q, s, v, act)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,K", SHAPES)
def test_norm(qc, M, K, t):
    import torch
    rng = np.random.default_rng(M + 3 * K)
    w = (1 + 0.2 * rng.standard_normal(K)).astype(np.float32)
    for residual, weight, place in ((True, True, "apart"), (False, True, "apart"), (True, False, "x"), (True, True, "residual"), (False, False, "apart")):
        x, xbuf = _rows(M, K, _type(t), 5, 2, _tokens(rng, M, K, t))
        r, rbuf = _rows(M, K, _type(t), 3, 1, _tokens(rng, M, K, t)) if residual else (None, None)
        want_h = (x.float() + r.float()).to(_type(t)) if residual else x.clone()
        h, hbuf = (None, None) if not residual else (x, xbuf) if place == "x" else (r, rbuf) if place == "residual" else _rows(M, K, _type(t), 1)
        y, ybuf = _rows(M, K, _type(t), 2, 1)
        q, qbuf = _rows(M, K, torch.int8, 3)
        s = torch.empty(M, device="cuda")
        qc.qc_t8_norm(x, q, s, weight=_dev(w) if weight else None, residual=r, h=h, y=y, eps=EPS)
        if residual:
            assert torch.equal(h, want_h) and _untouched(h, hbuf)
        v = O.norm(_np(want_h), w if weight else None, EPS)
        _same_codes(q, s, v, "%s residual %s weight %s" % (t, residual, weight))
        assert torch.equal(y.cpu(), torch.from_numpy(v).to(_type(t)))
        assert _untouched(q, qbuf) and _untouched(y, ybuf)
        # either result alone is the same
        y2, q2, s2 = torch.empty_like(y), torch.empty_like(q), torch.empty_like(s)
        qc.qc_t8_norm(want_h, weight=_dev(w) if weight else None, y=y2, eps=EPS)
        qc.qc_t8_norm(want_h, q2, s2, weight=_dev(w) if weight else None, eps=EPS)
        assert torch.equal(y, y2) and torch.equal(q, q2) and torch.equal(s, s2)


def test_norm_of_rows_that_are_not_finite(qc):
    import torch
    h = np.random.default_rng(1).standard_normal((6, 200)).astype(np.float32)
    h[1, 3], h[2, 4], h[3], h[4] = np.inf, np.nan, 0, 1e30
    q, s, y = torch.full((6, 200), 9, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda"), torch.empty((6, 200), device="cuda")
    qc.qc_t8_norm(_dev(h), q, s, y=y, eps=EPS)
    assert torch.isnan(s[1:3]).all() and torch.isfinite(s[[0, 3, 4, 5]]).all() and (q[1:3] == 0).all()
    assert (q[3] == 0).all() and s[3] == 1 and (y[3] == 0).all()
    v = O.norm(h[[0, 4, 5]], None, EPS)
    _same_codes(q[[0, 4, 5]], s[[0, 4, 5]], v, "finite rows")
    # float16 sums beyond the type are infinite, and their rows
    x = torch.full((2, 64), 6e4, dtype=torch.float16, device="cuda")
    x[1] = 1
    hh, q, s = torch.empty_like(x), torch.empty((2, 64), dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    qc.qc_t8_norm(x, q, s, residual=x, h=hh)
    assert torch.isinf(hh[0]).all() and torch.isnan(s[0]) and (hh[1] == 2).all() and (q[1] == 127).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,K", SHAPES)
def test_norm_grad(qc, M, K, t):
    import torch
    rng = np.random.default_rng(M + 5 * K)
    w = (1 + 0.2 * rng.standard_normal(K)).astype(np.float32)
    need = qc.qc_t8_norm_grad_bytes(M, K)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    for weight, add, place in ((True, True, "apart"), (True, False, "dy"), (False, True, "dh")):
        h, _ = _rows(M, K, _type(t), 3, 1, _tokens(rng, M, K, t))
        dy, dybuf = _rows(M, K, _type(t), 4, 3, _dev(rng.standard_normal((M, K))).to(_type(t)))
        dh, dhbuf = _rows(M, K, _type(t), 1, 0, _dev(rng.standard_normal((M, K))).to(_type(t))) if add else (None, None)
        hn, dyn, dhn = _np(h), _np(dy), None if dh is None else _np(dh)
        dx, buf = (dy, dybuf) if place == "dy" else (dh, dhbuf) if place == "dh" else _rows(M, K, _type(t), 2)
        dw = torch.empty(K, device="cuda")
        work.fill_(255)
        qc.qc_t8_norm_grad(h, dy, dx, weight=_dev(w) if weight else None, dh=dh, dweight=dw, work=work, eps=EPS)
        want, dww = O.norm_grad(hn, w if weight else None, EPS, dyn, dhn)
        r = O.rho(hn, EPS)[:, None]
        g = np.abs(dyn * (w if weight else 1.0))
        along = r ** 3 * np.abs(hn) / K
        tol = E * (4 * r * g + along * 8 * np.abs((dyn * (w if weight else 1.0) * hn).sum(1, keepdims=True)) + along * 33 * (g * np.abs(hn)).sum(1, keepdims=True))
        tol += 0 if dhn is None else E * np.abs(dhn)
        _check(dx, want, tol, t, "dx %s weight %s" % (t, weight))
        assert _untouched(dx, buf)
        n = -(-M // 512) * 4 + 8                   # rows of a group, four partial sums
        _check(dw, dww, (n + 4) * E * (np.abs(dyn * hn) * r).sum(0), "f32", "dweight")
        # without dweight no workspace is read
        dx2 = torch.empty_like(h)
        if place == "apart":
            qc.qc_t8_norm_grad(h, dy, dx2, weight=_dev(w), dh=dh, eps=EPS)
            assert torch.equal(dx2, dx)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,K", [s for s in SHAPES if s[0] * s[1] < 6e6])
def test_gated_grad(qc, M, K, t, act):
    import torch
    rng = np.random.default_rng(M + K)
    code = qc.QC_ACT_SILU if act == "silu" else qc.QC_ACT_GELU
    for place in ("apart", "in place"):
        x, xbuf = _rows(M, K, _type(t), 3, 1, _tokens(rng, M, K, t))
        g, gbuf = _rows(M, K, _type(t), 9, 4, _dev(rng.standard_normal((M, K)) * 3).to(_type(t)))
        d, _ = _rows(M, K, _type(t), 0, 0, _dev(rng.standard_normal((M, K))).to(_type(t)))
        xn, gn, dn = _np(x), _np(g), _np(d)
        dx, dg = (x, g) if place == "in place" else (_rows(M, K, _type(t), 2)[0], _rows(M, K, _type(t), 7, 2)[0])
        qc.qc_t8_gated_grad(x, g, d, dx, dg, act=code)
        wx, wg = O.gated_grad(xn, gn, act, dn)
        # the derivative's terms: the logistic function, and gate t' s (1 - s), which are of either sign
        s = 1 / (1 + np.exp(-gn)) if act == "silu" else 1 / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (gn + 0.044715 * gn ** 3)))
        slope = 1.0 if act == "silu" else 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * gn ** 2)
        _check(dx, wx, 16 * E * np.abs(wx) + 2.0 ** -149 * np.abs(dn), t, "dx %s %s" % (t, act))
        _check(dg, wg, (32 * E * (s + np.abs(gn) * slope * s * (1 - s)) + 2.0 ** -149 + 1e-12) * np.abs(dn * xn), t, "dgate %s %s" % (t, act))


# M, N, K
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("t", TYPES)
def test_gated_grad_of_far_gates(qc, t, act):
    """Gates on both sides of every case of the activation, beside ordinary ones and alone in their vectors, and gates that are not finite."""
    import torch
    code = qc.QC_ACT_SILU if act == "silu" else qc.QC_ACT_GELU
    sizes = [0.0, 2.0 ** -20, 0.3, 5.0, 8.9, 9.0, 9.1, 9.9, 10.5, 13.0, 14.1, 15.2, 30.0, 31.0, 68.5, 69.0, 69.5, 85.0, 90.0, 103.0, 104.5, 150.0, 210.0, 280.0, 400.0, 6e4]
    far = np.array([v for a in sizes for v in (a, -a)])
    rng = np.random.default_rng(5)
    K = 8 * len(far)
    gates = np.stack([np.repeat(far, 8), np.tile(far, 8)[rng.permutation(K)], np.where(np.arange(K) % 8 == 3, np.repeat(far, 8), rng.standard_normal(K))])
    x, d = [_dev(rng.standard_normal((3, K))).to(_type(t)) for _ in range(2)]
    g = _dev(gates).to(_type(t))
    gn = _np(g)
    dx, dg = torch.empty_like(x), torch.empty_like(x)
    qc.qc_t8_gated_grad(x, g, d, dx, dg, act=code)
    wx, wg = O.gated_grad(_np(x), gn, act, _np(d))
    # as above; results that are less than the least float32 are zero
    tt = gn if act == "silu" else 2 * np.sqrt(2 / np.pi) * (gn + 0.044715 * gn ** 3)
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-tt))
        o = 1 / (1 + np.exp(tt))
    slope = 1.0 if act == "silu" else 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * gn ** 2)
    with np.errstate(invalid="ignore"):
        along = np.nan_to_num(np.abs(gn) * slope * s * o)
    # float16 has nothing from 65520 on, the middle between its largest value, 65504, and 2^16: such results round to infinities
    over = (np.abs(wx) >= 65520) & (t == "f16")
    assert np.array_equal(_np(dx)[over], np.copysign(np.inf, wx[over]))
    fits = _dev(~over)
    wx = np.where(over, 0.0, wx)
    _check(torch.where(fits, dx, torch.zeros_like(dx)), wx, 16 * E * np.abs(wx) + 2.0 ** -149 * (1 + np.abs(_np(d))), t, "dx")
    _check(dg, wg, (32 * E * (s + along) + 2.0 ** -149 + 1e-12) * np.abs(_np(d) * _np(x)) + 2.0 ** -149, t, "dgate")
    # a gate that is not finite leaves its neighbours as they were
    for bad in (np.inf, -np.inf, np.nan):
        g2 = g.clone()
        g2[:, 5::16] = bad
        dx2, dg2 = torch.empty_like(x), torch.empty_like(x)
        qc.qc_t8_gated_grad(x, g2, d, dx2, dg2, act=code)
        same = torch.ones(K, dtype=torch.bool, device="cuda")
        same[5::16] = False
        dx2 = torch.where(fits | ~same, dx2, torch.zeros_like(dx2))
        _check(dx2[:, same], wx[:, _np(same) > 0], (16 * E * np.abs(wx) + 2.0 ** -149 * (1 + np.abs(_np(d))))[:, _np(same) > 0], t, "dx beside %s" % bad)
        if np.isnan(bad):
            assert torch.isnan(dx2[:, ~same]).all() and torch.isnan(dg2[:, ~same]).all()


PRODUCTS = [(1, 1, 16), (1, 17, 48), (2, 33, 144), (5, 100, 1168), (1, 700, 4608), (16, 48, 384), (17, 64, 272), (33, 31, 656), (64, 130, 1152),
            (77, 257, 1040), (128, 128, 128), (129, 200, 912), (300, 384, 1152), (513, 261, 400), (600, 300, 64), (1030, 515, 80), (1, 40, 14336),
            (2000, 1152, 208),
            # more tiles than workgroups, tiles of both sizes, ragged in every direction, one slab a tile, whole tiles
            (4090, 4085, 272), (9000, 4608, 144), (2500, 8000, 48), (5000, 5120, 128), (8192, 1000, 1152), (3, 9000, 352), (8100, 2300, 1152), (3000, 1500, 2320),
            # fewer tiles than compute units and a long summed axis, in either direction
            (900, 515, 4112), (1100, 1000, 1168), (800, 4100, 1040), (700, 2900, 1200), (30, 4100, 4096),
            # gradients whose rows are longer than a workgroup's registers, in all types and in float32 alone
            (5, 40000, 48), (40, 20000, 16),
            # whole tiles, and a rest whose summed axis is split: in 16-bit types and in float32
            (1851, 2965, 2208), (775, 2201, 2656)]


def _codes(rng, M, K, pad):
    import torch
    q, _ = _rows(M, K, torch.int8, 16 * pad, 16 if pad else 0, _dev(rng.integers(-128, 128, (M, K)).astype(np.int8)))
    return q if q.data_ptr() % 16 == 0 else q.contiguous()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_linear(qc, M, N, K, t):
    import torch
    rng = np.random.default_rng(M + N + K)
    for bias, pad in ((True, 0), (False, 3)):
        qx, qw = _codes(rng, M, K, pad), _codes(rng, N, K, pad)
        xs, ws = rng.uniform(0.001, 0.1, M).astype(np.float32), rng.uniform(0.0001, 0.01, N).astype(np.float32)
        b = rng.standard_normal(N).astype(np.float32)
        y, buf = _rows(M, N, _type(t), pad, min(pad, 1))
        qc.qc_t8_linear(qx, _dev(xs), qw, _dev(ws), y, bias=_dev(b) if bias else None)
        want = O.linear(_np(qx), xs, _np(qw), ws, b if bias else None)
        plain = O.linear(_np(qx), xs, _np(qw), ws)
        _check(y, want, 4 * E * (np.abs(plain) + (np.abs(b) if bias else 0)), t, "%s bias %s" % (t, bias))
        assert _untouched(y, buf)


def test_linear_exact_sums(qc):
    """Sums up to 2^31 of the most that codes can make, in the kernels of few and of many rows."""
    import torch
    for M, K in ((3, 131056), (600, 131056), (600, 2000 * 16)):
        qx = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
        qw = torch.full((20, K), -128, dtype=torch.int8, device="cuda")
        qw[1] = 127
        qx[1, ::2] = 127
        one = torch.ones(600, device="cuda")
        y = torch.empty((M, 20), device="cuda")
        qc.qc_t8_linear(qx, one[:M], qw, one[:20], y)
        want = (qx[:4].cpu().long() @ qw.cpu().long().t()).float()
        assert torch.equal(y[:4].cpu(), want), (M, K)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_linear_grad(qc, M, N, K, t):
    import torch
    rng = np.random.default_rng(M + N + K)
    for pad in (0, 3):
        dy, _ = _rows(M, N, _type(t), pad, min(pad, 1), _dev(rng.standard_normal((M, N)) * np.exp(rng.uniform(-6, 0, (M, 1)))).to(_type(t)))
        qw = _codes(rng, N, K, pad)
        ws = rng.uniform(0.0001, 0.01, N).astype(np.float32)
        dx, buf = _rows(M, K, _type(t), pad, min(pad, 1))
        work = torch.full((qc.qc_t8_linear_grad_bytes(M, N, K, _type(t)),), 255, dtype=torch.uint8, device="cuda")
        qc.qc_t8_linear_grad(dy, qw, _dev(ws), dx, work)
        want = O.linear_grad(_np(dy), _np(qw), ws)
        v = np.abs(_np(dy) * ws)
        step = 1.01 * 2.0 ** (-32 if t == "f32" else -16)
        aq = np.abs(_np(qw))
        tol = step * v.max(1, keepdims=True) * aq.sum(0) + 8 * E * (v @ aq)
        _check(dx, want, tol, t, t)
        assert _untouched(dx, buf)


def test_linear_grad_of_rows_that_are_not_finite_or_empty(qc):
    import torch
    rng = np.random.default_rng(8)
    for t in TYPES:
        dy = _dev(rng.standard_normal((40, 200))).to(_type(t))
        dy[3] = 0
        dy[5, 7], dy[6, 199] = float("inf"), float("nan")
        if t != "f16":
            dy[9] *= 1e-35
        qw, ws = _codes(rng, 200, 64, 0), torch.full((200,), 0.01, device="cuda")
        work = torch.empty(qc.qc_t8_linear_grad_bytes(40, 200, 64, _type(t)), dtype=torch.uint8, device="cuda")
        dx = torch.empty((40, 64), dtype=_type(t), device="cuda")
        qc.qc_t8_linear_grad(dy, qw, ws, dx, work)
        bad = torch.zeros(40, dtype=torch.bool, device="cuda")
        bad[5:7] = True
        assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all()
        assert (dx[3] == 0).all() and (t == "f16" or (dx[9] == 0).all())


def test_nothing_to_do(qc):
    """No rows, no outputs, no summed axis."""
    import torch
    e = lambda *s, d=torch.float32: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
    qc.qc_t8_quantize(e(0, 32), e(0, 32, d=torch.int8), e(0))
    qc.qc_t8_norm(e(0, 32), e(0, 32, d=torch.int8), e(0))
    qc.qc_t8_expand(e(0, 32, d=torch.int8), e(0), e(0, 32))
    qc.qc_t8_gated_grad(*[e(0, 32) for _ in range(5)])
    qc.qc_t8_linear(e(0, 32, d=torch.int8), e(0), e(5, 32, d=torch.int8), e(5), e(0, 5))
    qc.qc_t8_linear(e(4, 32, d=torch.int8), e(4), e(0, 32, d=torch.int8), e(0), e(4, 0))
    dw = torch.full((32,), 5.0, device="cuda")
    qc.qc_t8_norm_grad(e(0, 32), e(0, 32), e(0, 32), dweight=dw, work=e(16))
    assert (dw == 0).all()
    for t in TYPES:
        dx, buf = _rows(4, 32, _type(t), 3, 1)
        work = torch.empty(qc.qc_t8_linear_grad_bytes(4, 0, 32, _type(t)) + 16, dtype=torch.uint8, device="cuda")
        qc.qc_t8_linear_grad(e(4, 0, d=_type(t)), e(0, 32, d=torch.int8), e(0), dx, work)
        assert (dx == 0).all() and _untouched(dx, buf)
