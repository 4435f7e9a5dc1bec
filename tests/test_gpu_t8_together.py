"""The 8-bit layers with a scale for each token as they are used: one after the other on a stream, in graphs, on several streams, with one
workspace a call, beyond 32-bit offsets."""
import numpy as np
import pytest

from oracle import t8 as O
from test_gpu_t8 import E, EPS, HALF, _check, _dev, _np, _same_codes, _type, qc  # noqa: F401  (qc: the fixture)

pytestmark = pytest.mark.gpu


class Block:
    """Norm, gate | up projection, gated activation, down projection, and the next norm; its buffers and those of its gradients."""

    def __init__(self, qc, M, D, F, t, act, seed):
        import torch
        rng = np.random.default_rng(seed)
        self.qc, self.M, self.D, self.F, self.t, self.act = qc, M, D, F, t, act
        self.code = qc.QC_ACT_SILU if act == "silu" else qc.QC_ACT_GELU
        T = _type(t)
        new = lambda r, c, d=T: torch.empty((r, c), dtype=d, device="cuda")  # noqa: E731
        vec = lambda n: torch.empty(n, device="cuda")  # noqa: E731
        i8 = torch.int8
        # weights through the row quantiser: rows are output channels
        self.w1, self.s1, self.w2, self.s2 = new(2 * F, D, i8), vec(2 * F), new(D, F, i8), vec(D)
        qc.qc_t8_quantize(_dev(rng.standard_normal((2 * F, D)) / np.sqrt(D)).to(T), self.w1, self.s1)
        qc.qc_t8_quantize(_dev(rng.standard_normal((D, F)) / np.sqrt(F)).to(T), self.w2, self.s2)
        self.nw, self.nw2 = [_dev((1 + 0.2 * rng.standard_normal(D)).astype(np.float32)) for _ in range(2)]
        self.b1 = _dev((0.1 * rng.standard_normal(2 * F)).astype(np.float32))
        self.x, self.res, self.dy, self.dh = [_dev(rng.standard_normal((M, D))).to(T) for _ in range(4)]
        self.h, self.q1, self.x1 = new(M, D), new(M, D, i8), vec(M)
        self.gu, self.q2, self.x2 = new(M, 2 * F), new(M, F, i8), vec(M)
        self.o, self.h2, self.y = new(M, D), new(M, D), new(M, D)
        # gradients
        self.d_h2, self.d_act, self.d_gu, self.d_y1, self.dx = new(M, D), new(M, F), new(M, 2 * F), new(M, D), new(M, D)
        self.dw, self.dw2 = vec(D), vec(D)
        byte = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.wk_n = byte(qc.qc_t8_norm_grad_bytes(M, D))
        self.wk_2, self.wk_1 = byte(qc.qc_t8_linear_grad_bytes(M, D, F, T)), byte(qc.qc_t8_linear_grad_bytes(M, 2 * F, D, T))

    def inputs(self, seed):
        rng = np.random.default_rng(seed)
        for v in (self.x, self.res, self.dy, self.dh):
            v.copy_(_dev(rng.standard_normal((self.M, self.D))).to(v.dtype))

    def forward(self):
        qc, F = self.qc, self.F
        qc.qc_t8_norm(self.x, self.q1, self.x1, weight=self.nw, residual=self.res, h=self.h, eps=EPS)
        qc.qc_t8_linear(self.q1, self.x1, self.w1, self.s1, self.gu, bias=self.b1)
        qc.qc_t8_quantize(self.gu[:, F:], self.q2, self.x2, gate=self.gu[:, :F], act=self.code)
        qc.qc_t8_linear(self.q2, self.x2, self.w2, self.s2, self.o)
        qc.qc_t8_norm(self.o, weight=self.nw2, residual=self.h, h=self.h2, y=self.y, eps=EPS)

    def backward(self):
        qc, F = self.qc, self.F
        qc.qc_t8_norm_grad(self.h2, self.dy, self.d_h2, weight=self.nw2, dh=self.dh, dweight=self.dw2, work=self.wk_n, eps=EPS)
        qc.qc_t8_linear_grad(self.d_h2, self.w2, self.s2, self.d_act, self.wk_2)
        qc.qc_t8_gated_grad(self.gu[:, F:], self.gu[:, :F], self.d_act, self.d_gu[:, F:], self.d_gu[:, :F], act=self.code)
        qc.qc_t8_linear_grad(self.d_gu, self.w1, self.s1, self.d_y1, self.wk_1)
        qc.qc_t8_norm_grad(self.h, self.d_y1, self.dx, weight=self.nw, dh=self.d_h2, dweight=self.dw, work=self.wk_n, eps=EPS)

    RESULTS = ("h", "q1", "x1", "gu", "q2", "x2", "o", "h2", "y", "d_h2", "d_act", "d_gu", "d_y1", "dx", "dw", "dw2")

    def results(self):
        return {k: getattr(self, k).clone() for k in self.RESULTS}

    def check(self):
        """Every step from the values that the one before it left."""
        F, t = self.F, self.t
        n = lambda v: _np(v)  # noqa: E731
        h = (self.x.float() + self.res.float()).to(_type(t))
        assert (h == self.h).all()
        _same_codes(self.q1, self.x1, O.norm(n(self.h), n(self.nw), EPS), "first codes")
        lin = lambda q, xs, w, s, b=None: O.linear(n(q), n(xs), n(w), n(s), b)  # noqa: E731
        plain = lin(self.q1, self.x1, self.w1, self.s1)
        _check(self.gu, plain + n(self.b1), 4 * E * (np.abs(plain) + np.abs(n(self.b1))), t, "gate | up")
        g, u = n(self.gu[:, :F]), n(self.gu[:, F:])
        _same_codes(self.q2, self.x2, O.gated(u, g, self.act), "second codes")
        plain = lin(self.q2, self.x2, self.w2, self.s2)
        _check(self.o, plain, 4 * E * np.abs(plain), t, "down")
        assert ((self.o.float() + self.h.float()).to(_type(t)) == self.h2).all()
        y = O.norm(n(self.h2), n(self.nw2), EPS)
        _check(self.y, y, 0, t, "normalised")
        self._norm_grad(self.h2, self.nw2, self.dy, self.dh, self.d_h2, self.dw2, "second norm")
        self._linear_grad(self.d_h2, self.w2, self.s2, self.d_act, "down")
        wx, wg = O.gated_grad(u, g, self.act, n(self.d_act))
        s = O.act(self.act, np.abs(g))[1] + 1                   # the derivative's terms, in all
        _check(self.d_gu[:, F:], wx, 16 * E * np.abs(wx), t, "d up")
        _check(self.d_gu[:, :F], wg, 64 * E * s * np.abs(n(self.d_act) * u), t, "d gate")
        self._linear_grad(self.d_gu, self.w1, self.s1, self.d_y1, "gate | up")
        self._norm_grad(self.h, self.nw, self.d_y1, self.d_h2, self.dx, self.dw, "first norm")

    def _norm_grad(self, h, w, dy, dh, dx, dw, what):
        hn, g, r = _np(h), _np(dy) * _np(w), O.rho(_np(h), EPS)[:, None]
        want, dww = O.norm_grad(hn, _np(w), EPS, _np(dy), _np(dh))
        tol = E * (4 * r * np.abs(g) + r ** 3 * np.abs(hn) / self.D * (33 * np.abs(g * hn).sum(1, keepdims=True) + 8 * np.abs((g * hn).sum(1, keepdims=True)))
                   + np.abs(_np(dh)))
        _check(dx, want, tol, self.t, what)
        _check(dw, dww, (self.M / 128 + 16) * E * (np.abs(_np(dy) * hn) * r).sum(0), "f32", what + ", weight")

    def _linear_grad(self, dy, w, s, dx, what):
        v, aq = np.abs(_np(dy) * _np(s)), np.abs(_np(w))
        step = 1.01 * 2.0 ** (-32 if self.t == "f32" else -16)
        _check(dx, O.linear_grad(_np(dy), _np(w), _np(s)), step * v.max(1, keepdims=True) * aq.sum(0) + 8 * E * (v @ aq), self.t, what)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,D,F,act", [(1, 128, 352, "silu"), (77, 1152, 304, "gelu"), (700, 400, 1168, "silu")])
def test_a_block_forwards_and_backwards(qc, M, D, F, t, act):  # noqa: F811
    b = Block(qc, M, D, F, t, act, M + D)
    b.forward()
    b.backward()
    b.check()


def test_a_block_on_another_stream_and_in_graphs(qc):  # noqa: F811
    """Two blocks, each captured, replayed by turns with new inputs and eager work between the replays: every replay is the eager result."""
    import torch
    side = torch.cuda.Stream()
    blocks = [Block(qc, 300, 256, 400, "bf16", "silu", 1), Block(qc, 33, 512, 176, "f32", "gelu", 2)]
    eager = [Block(qc, 300, 256, 400, "bf16", "silu", 1), Block(qc, 33, 512, 176, "f32", "gelu", 2)]
    graphs = []
    for b in blocks:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b.forward()
            b.backward()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.forward()
            b.backward()
        graphs.append(g)
    for turn in range(4):
        for b, e, g in zip(blocks, eager, graphs):
            b.inputs(10 * turn + b.M)
            e.inputs(10 * turn + b.M)
            g.replay()
            e.forward()
            e.backward()
        if turn % 2:
            torch.cuda.synchronize()
        for b, e in zip(blocks, eager):
            want = e.results()
            for k, v in b.results().items():
                assert torch.equal(v, want[k]), (turn, k)
    blocks[0].check()


def test_calls_of_two_streams_at_once(qc):  # noqa: F811
    import torch
    streams = [torch.cuda.Stream() for _ in range(2)]
    blocks = [Block(qc, 2000, 640, 960, "f16", "silu", s) for s in (5, 6)]
    want = []
    for b in blocks:
        b.forward()
        b.backward()
        want.append(b.results())
        for k in Block.RESULTS:
            getattr(b, k).zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for s, b in zip(streams, blocks):
            with torch.cuda.stream(s):
                b.forward()
                b.backward()
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        for k, v in b.results().items():
            assert torch.equal(v, w[k]), k


def test_the_weight_quantiser_gives_the_same(qc):  # noqa: F811
    """qc_quantize_weight's codes and scales go into the product as they are."""
    import torch
    w = torch.randn((200, 272), device="cuda")
    a, s, wsum = torch.empty((200, 272), dtype=torch.int8, device="cuda"), torch.empty(200, device="cuda"), torch.empty(200, dtype=torch.int32, device="cuda")
    qc.qc_quantize_weight(w, 8, a, s, wsum)
    b, t = torch.empty_like(a), torch.empty_like(s)
    qc.qc_t8_quantize(w, b, t)
    assert torch.equal(a, b) and torch.equal(s, t)


@pytest.mark.parametrize("t", ["f16", "f32"])
def test_millions_of_short_rows(qc, t):  # noqa: F811
    """More workgroups than one dimension of a grid takes."""
    import torch
    M, K = 4300003, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((M, K), generator=g, device="cuda").to(_type(t))
    q, s, out = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda"), torch.empty_like(x)
    qc.qc_t8_quantize(x, q, s)
    qc.qc_t8_expand(q, s, out)
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(K, device="cuda")
    qc.qc_t8_norm(x, y=y, eps=EPS)
    work = torch.empty(qc.qc_t8_norm_grad_bytes(M, K), dtype=torch.uint8, device="cuda")
    qc.qc_t8_norm_grad(x, x, dx, dweight=dw, work=work, eps=EPS)
    want = x.float().abs().amax(1) / torch.full((), 127.0, device="cuda")
    assert torch.equal(s, want)
    assert torch.equal(q.float(), torch.round(x.float() / s[:, None]).clamp(-127, 127))
    assert torch.equal(out, (q.float() * s[:, None]).to(x.dtype))
    rho = (1 / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + EPS))
    assert torch.equal(y, (x.float() * rho.float()).to(x.dtype))
    total = (x.double() ** 2 * rho).sum(0)
    assert ((dw.double() - total).abs() <= (M / 128 + 16) * E * total).all()


def test_offsets_beyond_32_bits(qc):  # noqa: F811
    """Tensors of more than 2^32 bytes, of codes too: the last rows are like the first."""
    import torch
    M, K, N = 140000, 32768, 64
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    last = torch.randn((300, K), device="cuda").to(torch.bfloat16)
    x.zero_()
    x[-300:] = last
    x[:300] = last
    q, s = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    qc.qc_t8_quantize(x, q, s)
    _same_codes(q[-300:], s[-300:], _np(last).astype(np.float32), "last rows")
    assert torch.equal(q[:300], q[-300:]) and (s[300:-300] == 1).all() and (q[700] == 0).all()
    w, ws = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda"), torch.full((N,), 0.01, device="cuda")
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    qc.qc_t8_linear(q, s, w, ws, y)
    assert torch.equal(y[:300], y[-300:]) and (y[300:-300] == 0).all()
    plain = O.linear(_np(q[-300:]), _np(s[-300:]), _np(w), _np(ws))
    _check(y[-300:], plain, 4 * E * np.abs(plain), "bf16", "last rows")
    # the residual stream in place, and the norm's gradient in place of dy
    qc.qc_t8_norm(x, q, s, residual=x, h=x, eps=EPS)
    assert torch.equal(x[-300:], (last.float() * 2).to(torch.bfloat16)) and torch.equal(q[:300], q[-300:])
    _same_codes(q[-300:], s[-300:], O.norm(_np(x[-300:]), None, EPS), "normalised")
    dy = x.clone()
    qc.qc_t8_norm_grad(x, dy, dy, eps=EPS)
    assert torch.equal(dy[:300], dy[-300:]) and (dy[300:-300] == 0).all()
    qc.qc_t8_gated_grad(x, x, dy, dy, x)
    assert torch.equal(x[:300], x[-300:]) and torch.equal(dy[:300], dy[-300:])


def test_a_gradient_whose_planes_pass_32_bits(qc):  # noqa: F811
    import torch
    M, N, K = 1100000, 2048, 32
    dy = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    rows = torch.randn((200, N), device="cuda").to(torch.bfloat16)
    dy[:200] = rows
    dy[-200:] = rows
    w, ws = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda"), torch.full((N,), 0.01, device="cuda")
    work = torch.empty(qc.qc_t8_linear_grad_bytes(M, N, K, torch.bfloat16), dtype=torch.uint8, device="cuda")
    assert work.numel() > 1 << 32
    dx = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    qc.qc_t8_linear_grad(dy, w, ws, dx, work)
    assert torch.equal(dx[:200], dx[-200:]) and (dx[200:-200] == 0).all()
    v, aq = np.abs(_np(rows) * 0.01), np.abs(_np(w))
    _check(dx[-200:], O.linear_grad(_np(rows), _np(w), _np(ws)), 1.01 * 2.0 ** -16 * v.max(1, keepdims=True) * aq.sum(0) + 8 * E * (v @ aq), "bf16", "last rows")


def test_a_result_beyond_32_bits(qc):  # noqa: F811
    import torch
    M, N, K = 600001, 4100, 64
    q = torch.zeros((M, K), dtype=torch.int8, device="cuda")
    rows = torch.randint(-127, 128, (150, K), dtype=torch.int8, device="cuda")
    q[:150] = rows
    q[-150:] = rows
    s, ws = torch.full((M,), 0.5, device="cuda"), torch.full((N,), 0.25, device="cuda")
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda")
    y = torch.empty((M, N), dtype=torch.float16, device="cuda")
    qc.qc_t8_linear(q, s, w, ws, y)
    want = ((rows.double() @ w.double().t()) * 0.125).to(torch.float16)
    assert torch.equal(y[:150], want) and torch.equal(y[-150:], want) and (y[150:-150] == 0).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_gradients_against_differences(qc, t):  # noqa: F811
    """The float64 functions' central differences along a random direction, against the kernels' gradients: the differences' error is 1e-8
    of the sum of magnitudes, the gradients' half a step of their type and 40 e of theirs."""
    import torch
    rng = np.random.default_rng(9)
    M, K = 5, 200
    x, g, d, way, way2 = [_np(_dev(rng.standard_normal((M, K))).to(_type(t))) for _ in range(5)]
    put = lambda a: _dev(a).to(_type(t))  # noqa: E731
    dx, dg = torch.empty((M, K), dtype=_type(t), device="cuda"), torch.empty((M, K), dtype=_type(t), device="cuda")
    h = 1e-5
    for act, code in (("silu", qc.QC_ACT_SILU), ("gelu", qc.QC_ACT_GELU)):
        qc.qc_t8_gated_grad(put(x), put(g), put(d), dx, dg, act=code)
        f = lambda e: float((d * O.act(act, g + e * way2)[0] * (x + e * way)).sum())  # noqa: E731
        want = (f(h) - f(-h)) / (2 * h)
        size = np.abs(_np(dx) * way).sum() + np.abs(_np(dg) * way2).sum()
        assert abs((_np(dx) * way).sum() + (_np(dg) * way2).sum() - want) <= (1e-8 + HALF[t] + 40 * E) * size
    w = (1 + 0.2 * rng.standard_normal(K)).astype(np.float32)
    dw = torch.empty(K, device="cuda")
    work = torch.empty(qc.qc_t8_norm_grad_bytes(M, K), dtype=torch.uint8, device="cuda")
    qc.qc_t8_norm_grad(put(x), put(d), dx, weight=_dev(w), dweight=dw, work=work, eps=EPS)
    wway = rng.standard_normal(K)

    def f(e):
        v = x + e * way
        return float((d * v * O.rho(v, EPS)[:, None] * (w + e * wway)).sum())

    size = np.abs(_np(dx) * way).sum() + np.abs(_np(dw) * wway).sum()
    assert abs((_np(dx) * way).sum() + (_np(dw) * wway).sum() - (f(h) - f(-h)) / (2 * h)) <= (1e-8 + HALF[t] + 40 * E) * size
