"""8-bit layers with a scale for each token (include/qc_t8.h) on values of very different sizes, against the float64 oracle: outliers within a row,
the ends of the types' ranges.  (e = 2^-24, half a float32 step; helpers and the other tolerances: test_gpu_t8.py)"""
import numpy as np
import pytest

from oracle import t8 as O
from test_gpu_t8 import E, EPS, PRODUCTS, _check, _dev, _np, _rows, _same_codes, _type, _untouched, qc  # noqa: F401  (qc: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_linear_grad_beside_an_outlier(qc, M, N, K, t):  # noqa: F811
    """One gradient of a row a thousand times the others, and columns that it does not reach (its weights there are 0): what is left there are the
    others.  A term dy w_s is a float32 product (e of itself) and a number of 24 bits of its row's largest (half a step of 1 / (127 2^16): 1.01 e
    of the largest); the integer sum and its float64 product with the scale are off by the scale's e: 4 e of the terms are counted."""
    import torch
    rng = np.random.default_rng(M + 2 * N + 3 * K)
    dy = 0.01 * rng.standard_normal((M, N))
    qw = rng.integers(-128, 128, (N, K)).astype(np.int8)
    out = int(rng.integers(0, N))
    dy[:, out] *= 1000
    qw[out, rng.permutation(K)[:K // 2]] = 0
    ws = rng.uniform(0.005, 0.01, N).astype(np.float32)
    d, _ = _rows(M, N, _type(t), 3, 1, _dev(dy).to(_type(t)))
    dx, buf = _rows(M, K, _type(t), 5, 2)
    work = torch.full((qc.qc_t8_linear_grad_bytes(M, N, K, _type(t)),), 255, dtype=torch.uint8, device="cuda")
    qc.qc_t8_linear_grad(d, _dev(qw), _dev(ws), dx, work)
    v, aq = np.abs(_np(d) * ws), np.abs(qw.astype(np.float64))
    _check(dx, O.linear_grad(_np(d), qw, ws), 1.01 * E * v.max(1, keepdims=True) * aq.sum(0) + 4 * E * (v @ aq), t, t)
    assert _untouched(dx, buf)


def _gated(qc, x, g, act, t):
    """Codes and scales of rows, against the oracle's."""
    import torch
    xt, gt = _dev(x).to(_type(t)), _dev(g).to(_type(t))
    q, s = torch.full(x.shape, 55, dtype=torch.int8, device="cuda"), torch.empty(len(x), device="cuda")
    qc.qc_t8_quantize(xt, q, s, gate=gt, act=qc.QC_ACT_SILU if act == "silu" else qc.QC_ACT_GELU)
    with np.errstate(over="ignore"):
        _same_codes(q, s, O.gated(_np(xt), _np(gt), act), "%s %s" % (act, t))
    return s


# a wavefront a row, one vector a lane and four; a workgroup a row; rows that are read again
GATED_WIDTHS = [64, 300, 1000, 4608, 40000]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("K", GATED_WIDTHS)
def test_gates_at_the_types_lowest_value_beside_ordinary_ones(qc, K, act, t):  # noqa: F811
    """act(gate) is 0 or next to it whatever x is: what such an element makes of its row is nothing."""
    import torch
    rng = np.random.default_rng(K)
    rows = 2100 if K == 300 else 9                           # (2100: one wavefront a row whatever the width)
    x, g = rng.standard_normal((rows, K)), rng.standard_normal((rows, K))
    lowest = float(torch.finfo(_type(t)).min)
    at = rng.integers(0, K, rows)
    far = [(lowest, 1.0), (lowest, 3e38), (-1e36, 1.0), (-1e38, 1e38), (-100.0, 3e38), (-100.0, -1e36), (-86.0, 1e37), (-20.0, 3e38)]
    for m in range(rows - 1):                                 # the last row has none
        g[m, at[m]], x[m, at[m]] = far[m % len(far)]
    g[0, K // 2:] = lowest                                    # a masked half
    s = _gated(qc, x, g, act, t)
    assert torch.isfinite(s).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("K", GATED_WIDTHS)
def test_gated_rows_of_subnormal_factors(qc, K, act, t):  # noqa: F811
    """Products of a subnormal gate (or row) and a large factor: a float32 product that is rounded on its way among the subnormal numbers has lost its
    digits when the other factor brings it back."""
    rng = np.random.default_rng(K + 1)
    step = 2.0 ** (-149 if t == "f32" else -133)              # the type's least number
    x, g = rng.standard_normal((12, K)), rng.standard_normal((12, K))
    at = rng.integers(0, K // 2, 12)
    for m, (size, gate, factor) in enumerate([(1e-14, 3, 2.0 ** 127), (1e-14, 1, 2.0 ** 127), (1e-14, -5, 2.0 ** 127), (1e-15, 7, -2.0 ** 125), (0, 1, 2.0 ** 127),
                                              (1e-12, 11, 2.0 ** 127)]):
        x[m] *= size if t == "f32" else size * 2.0 ** 16
        g[m, at[m]], x[m, at[m]] = gate * step, factor
    # rows of nothing but subnormal products: gates, then rows
    g[6], x[6] = np.round(g[6] * 1000) * step, x[6] * 1000
    g[7], x[7] = np.round(g[7] * 30) * step, 2.0 ** 20
    g[8], x[8] = g[8] * 8, np.round(x[8] * 1000) * step
    # two elements that are nearly the largest: which one is, the nearer of the approximations does not know
    if t == "f32":
        for m, (a, b) in ((9, ((1001 * step, 1024.0), (100.0, 5122 * step))), (10, ((9.0, 4086 * step), (36766.0, step))),
                             (11, ((3.5, 3103 * step), (10858.0, step)))):
            x[m] = 0
            g[m, at[m]], x[m, at[m]] = a
            g[m, K - 2], x[m, K - 2] = b
    _gated(qc, x, g, act, t)


@pytest.mark.parametrize("N", [3, 5, 40, 700, 20000])
def test_linear_grad_of_small_float32_rows(qc, N):  # noqa: F811
    """Rows whose largest dy w_s lies between 2^-100, below which they may be zeros, and 2^-94.  No term is of another sign than the others, so
    that the result's error is its terms': a float32 product (e), 32 bits of the row's largest, the scale and the last product (4 e)."""
    import torch
    rng = np.random.default_rng(N)
    M, K = 300, 48
    dy = rng.uniform(0.5, 1, (M, N)) * 2.0 ** rng.uniform(-99, -94, (M, 1))
    ws = np.ones(N, np.float32)
    qw = rng.integers(1, 128, (N, K)).astype(np.int8)
    d, dx = _dev(dy.astype(np.float32)), torch.empty((M, K), device="cuda")
    work = torch.empty(qc.qc_t8_linear_grad_bytes(M, N, K, torch.float32), dtype=torch.uint8, device="cuda")
    qc.qc_t8_linear_grad(d, _dev(qw), _dev(ws), dx, work)
    v, aq = _np(d), qw.astype(np.float64)
    _check(dx, O.linear_grad(v, qw, ws), 1.01 * 2.0 ** -32 * v.max(1, keepdims=True) * aq.sum(0) + 4 * E * (v @ aq), "f32", "N %d" % N)


def _norm_grad(qc, hn, dyn, w, t):
    """dx and dweight of qc_t8_norm_grad against the oracle's, by the bounds of test_norm_grad."""
    import torch
    M, K = hn.shape
    h, dy = _dev(hn).to(_type(t)), _dev(dyn).to(_type(t))
    dx, dw = torch.empty_like(h), torch.empty(K, device="cuda")
    work = torch.empty(qc.qc_t8_norm_grad_bytes(M, K), dtype=torch.uint8, device="cuda")
    qc.qc_t8_norm_grad(h, dy, dx, weight=_dev(w), dweight=dw, work=work, eps=EPS)
    hn, dyn = _np(h), _np(dy)
    want, dww = O.norm_grad(hn, w, EPS, dyn)
    r = O.rho(hn, EPS)[:, None]
    g = np.abs(dyn * w)
    along = r ** 3 * np.abs(hn) / K
    gh = dyn * w * hn
    _check(dx, want, E * (4 * r * g + along * 8 * np.abs(gh.sum(1, keepdims=True)) + along * 33 * np.abs(gh).sum(1, keepdims=True)), t, "dx")
    _check(dw, dww, (M + 8) * E * (np.abs(dyn * hn) * r).sum(0), "f32", "dweight")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", [(9, 5), (9, 64), (300, 1153), (9, 4608), (5, 9001), (3, 20000)])
def test_norm_grad_of_large_rows(qc, M, K, t):  # noqa: F811
    """Rows of 1e15 to 1e32, gradients along them (what is left is a hundredth of the two terms) and across them: rho^3 mean(g h) is below any float32 there,
    its product with h is not."""
    rng = np.random.default_rng(M + K)
    u = rng.standard_normal((M, K))
    size = 10.0 ** np.linspace(15, 32, M)[:, None]
    u /= np.abs(u).max(1, keepdims=True)
    dy = u + 0.01 * rng.standard_normal((M, K))
    dy[::3] = rng.standard_normal(dy[::3].shape)
    _norm_grad(qc, u * size, dy * 1e3, (1 + 0.2 * rng.standard_normal(K)).astype(np.float32), t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", [(9, 5), (9, 64), (300, 1153), (9, 4608), (5, 9001), (3, 20000)])
def test_norm_grad_of_large_rows_and_gradients(qc, M, K, t):  # noqa: F811
    """Products g h beyond float32, their sums of either size: results that are ordinary numbers."""
    rng = np.random.default_rng(M + 2 * K)
    h, dy = rng.standard_normal((M, K)), rng.standard_normal((M, K))
    _norm_grad(qc, h * 10.0 ** np.linspace(18, 36, M)[:, None], dy * 10.0 ** np.linspace(28, 20, M)[:, None], (1 + 0.2 * rng.standard_normal(K)).astype(np.float32), t)
