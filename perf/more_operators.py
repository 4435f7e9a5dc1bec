"""Performance cases of the 8-bit layers with a scale for each token (include/qc_t8.h).

Six operators on rows of float32, float16 or bfloat16 (tokens):
  norm         h = x + residual, rounded to the type; root-mean-square norm of h with a weight; rows of 8-bit codes with a scale
               each, returned as the values that they stand for, beside h and the scales
  norm_grad    its gradient: dx = d(residual), and the weight's, from the gradients of the normalised rows and of h
  quantize     rows, or rows times an activation of their gates, to 8-bit codes with a scale each, returned as values
  gated_grad   gradients of the rows and of the gates
  linear       y = x W^T + b of 8-bit codes, with a scale for every row of x and for every row of W
  linear_grad  dx = dy W through such a W

Codes of a row v (float32): scale = max |v| / 127, or 1 where that is 0; round(v / scale), half to even, in -127..127; the quotients
are float32 divisions.  In `norm` v = (h rho) w in two float32 products, rho the float32 rounding of 1 / sqrt(mean h^2 + eps)."""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
ACTS = {"silu": 0, "gelu": 1}
EPS = float(np.float32(1e-6))


def _case(name, op, M, N, K, dtype, act="none", add=False):
    """act: activation of the gates ("none": no gates); add: a residual (norm), a gradient of h (norm_grad), a bias (linear)."""
    c = {"op": op, "M": M, "N": N, "K": K, "dtype": dtype, "act": act, "add": add}
    return {"name": name, **c} if name else c


def listed():
    return [
        # serving, a single token of a wide model: latency
        _case("norm 1x8192 bf16", "norm", 1, 0, 8192, "bf16", add=True),
        # the tokens of 64 images of 256 tokens, width 1152, with the residual stream
        _case("norm 16384x1152 bf16", "norm", 16384, 0, 1152, "bf16", add=True),
        # training: an odd width, float32; a long batch with the gradient that arrives along the residual stream
        _case("norm_grad 1000x1153 f32", "norm_grad", 1000, 0, 1153, "f32"),
        _case("norm_grad 8192x4096 bf16", "norm_grad", 8192, 0, 4096, "bf16", add=True),
        # inputs of a second product: a few odd rows in float32; the gated activations of 64 images
        _case("quantize 77x4608 f32", "quantize", 77, 0, 4608, "f32"),
        _case("quantize gated 16384x4608 bf16", "quantize", 16384, 0, 4608, "bf16", act="silu"),
        # training the gated block of 16 images; a ragged float32 batch
        _case("gated_grad 4096x4608 f16", "gated_grad", 4096, 0, 4608, "f16", act="gelu"),
        _case("gated_grad 515x3081 f32", "gated_grad", 515, 0, 3081, "f32", act="silu"),
        # a single token through a large layer: the weights' bytes are all there is
        _case("linear 1 row bf16", "linear", 1, 28672, 8192, "bf16"),
        # the refresh step of 64 images of 256 tokens: first MLP matrix
        _case("linear 16384 rows bf16", "linear", 16384, 4608, 1152, "bf16", add=True),
        # gradients through fixed weights: an odd number of rows, float32; 32 images
        _case("linear_grad 1001 rows f32", "linear_grad", 1001, 1152, 4608, "f32"),
        _case("linear_grad 8192 rows bf16", "linear_grad", 8192, 4608, 1152, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "quantize", "gated_grad", "linear", "linear", "linear_grad"])
    c = _case("", op, 1, 0, 1, rng.choice(["f32", "f16", "bf16"]), add=rng.random() < 0.5)
    if op == "gated_grad" or (op == "quantize" and rng.random() < 0.5):
        c["act"] = rng.choice(["silu", "gelu"])
    while True:
        c["M"] = _log_int(rng, 1, 16384)
        if op in ("linear", "linear_grad"):
            c["N"], c["K"] = _log_int(rng, 64, 28672), 16 * _log_int(rng, 8, 896)
        else:
            c["K"] = _log_int(rng, 64, 16384)
        w = work(c)
        if w["flops"] <= 1.7e11 and w["bytes"] <= 4.0e8:
            return c


# ---------------------------------------------------------------- inputs
def _codes_of(v):
    """Codes and scales of float32 rows."""
    scale = v.abs().amax(1) / torch.full((), 127.0, device=v.device)
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    return torch.round(v / scale[:, None]).clamp(-127, 127), scale


def _buffer_of_codes(M, K, dev):
    """Rows of codes start at multiples of 16 bytes."""
    return torch.empty((M, -(-K // 16) * 16), dtype=torch.int8, device=dev)[:, :K]


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    M, N, K, t = c["M"], c["N"], c["K"], TYPES[c["dtype"]]
    s = SimpleNamespace(case=c)
    rnd = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    # tokens differ in size, and a few features are much larger than the others
    feature = 1 + 7 * (torch.rand((1, K), generator=g, device=dev) < 0.01).float()
    size = lambda: 0.5 + torch.rand((M, 1), generator=g, device=dev)  # noqa: E731
    if c["op"] in ("linear", "linear_grad"):
        w, s.ws = _codes_of(rnd(N, K) / math.sqrt(K) * (1 + 0.5 * torch.rand((N, 1), generator=g, device=dev)))
        s.w = w.to(torch.int8)
    if c["op"] == "linear":
        x, s.xs = _codes_of(rnd(M, K) * feature * size())
        s.x = x.to(torch.int8)
        s.b = 0.1 * rnd(N) if c["add"] else None
        s.y = torch.empty((M, N), dtype=t, device=dev)
    elif c["op"] == "linear_grad":
        s.dy = (0.01 * rnd(M, N) * size()).to(t)
        s.dx = torch.empty((M, K), dtype=t, device=dev)
        if own:
            import paper_2503_02508_amd as qc
            s.work = torch.empty(qc.qc_t8_linear_grad_bytes(M, N, K, t), dtype=torch.uint8, device=dev)
    elif c["op"] == "norm":
        s.x = (rnd(M, K) * size()).to(t)
        s.r = (rnd(M, K) * feature).to(t) if c["add"] else None
        s.w = 1 + 0.1 * rnd(K)
        s.h = torch.empty((M, K), dtype=t, device=dev) if c["add"] else None
    elif c["op"] == "norm_grad":
        s.h = (rnd(M, K) * feature * size()).to(t)
        s.dy = (0.01 * rnd(M, K)).to(t)
        s.dh = (0.01 * rnd(M, K)).to(t) if c["add"] else None
        s.w = 1 + 0.1 * rnd(K)
        s.dx, s.dw = torch.empty((M, K), dtype=t, device=dev), torch.empty((K,), device=dev)
        if own:
            import paper_2503_02508_amd as qc
            s.work = torch.empty(qc.qc_t8_norm_grad_bytes(M, K), dtype=torch.uint8, device=dev)
    else:
        s.x = (rnd(M, K) * size()).to(t)
        s.gate = rnd(M, K).to(t) if c["act"] != "none" else None
        if c["op"] == "gated_grad":
            s.dh = (0.01 * rnd(M, K)).to(t)
            s.dx, s.dg = torch.empty((M, K), dtype=t, device=dev), torch.empty((M, K), dtype=t, device=dev)
    if c["op"] in ("norm", "quantize"):
        s.q, s.scale = _buffer_of_codes(M, K, dev), torch.empty((M,), device=dev)
        s.out = torch.empty((M, K), dtype=t, device=dev)
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2503_02508_amd as qc
    c = s.case
    op = c["op"]
    if op == "norm":
        qc.qc_t8_norm(s.x, q=s.q, scale=s.scale, weight=s.w, residual=s.r, h=s.h, eps=EPS)
        qc.qc_t8_expand(s.q, s.scale, s.out)
        return [s.out, s.scale] + ([s.h] if c["add"] else [])
    if op == "quantize":
        qc.qc_t8_quantize(s.x, s.q, s.scale, gate=s.gate, act=ACTS.get(c["act"], 0))
        qc.qc_t8_expand(s.q, s.scale, s.out)
        return [s.out, s.scale]
    if op == "norm_grad":
        qc.qc_t8_norm_grad(s.h, s.dy, s.dx, weight=s.w, dh=s.dh, dweight=s.dw, work=s.work, eps=EPS)
        return [s.dx, s.dw]
    if op == "gated_grad":
        qc.qc_t8_gated_grad(s.x, s.gate, s.dh, s.dx, s.dg, act=ACTS[c["act"]])
        return [s.dx, s.dg]
    if op == "linear":
        qc.qc_t8_linear(s.x, s.xs, s.w, s.ws, s.y, bias=s.b)
        return [s.y]
    qc.qc_t8_linear_grad(s.dy, s.w, s.ws, s.dx, s.work)
    return [s.dx]


def _act(name, v):
    """Value and derivative."""
    if name == "silu":
        e = 1 / (1 + torch.exp(-v))
        return v * e, e * (1 + v * (1 - e))
    a, b = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(a * (v + b * v * v * v))
    return 0.5 * v * (1 + t), 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * a * (1 + 3 * b * v * v)


def _rho(h):
    return (1 / torch.sqrt((h.double() * h.double()).mean(1, keepdim=True) + EPS)).float()


def _run_plain(s):
    c = s.case
    op, t = c["op"], TYPES[c["dtype"]]
    if op == "norm":
        h = (s.x.float() + s.r.float()).to(t) if c["add"] else s.x
        q, scale = _codes_of(h.float() * _rho(h) * s.w)
        return [(q * scale[:, None]).to(t), scale] + ([h] if c["add"] else [])
    if op == "quantize":
        # values next to a border between two codes: 64 bits, rounded once to float32
        v = s.x.float() if s.gate is None else (_act(c["act"], s.gate.double())[0] * s.x.double()).float()
        q, scale = _codes_of(v)
        return [(q * scale[:, None]).to(t), scale]
    if op == "norm_grad":
        h, dy, rho = s.h.float(), s.dy.float(), _rho(s.h)
        n, dn = h * rho, dy * s.w
        dx = rho * (dn - n * (dn * n).mean(1, keepdim=True))
        if c["add"]:
            dx = dx + s.dh.float()
        return [dx.to(t), (dy * n).sum(0)]
    if op == "gated_grad":
        a, d = _act(c["act"], s.gate.float())
        dh = s.dh.float()
        return [(dh * a).to(t), (dh * s.x.float() * d).to(t)]
    if op == "linear":
        y = (s.x.float() @ s.w.float().t()) * s.xs[:, None] * s.ws
        return [(y + s.b if c["add"] else y).to(t)]
    return [((s.dy.float() * s.ws) @ s.w.float()).to(t)]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    M, N, K, e = c["M"], c["N"], c["K"], BYTES[c["dtype"]]
    # codes are written, and read again as the values they stand for
    codes = M * K * (1 + 1 + e) + 8 * M
    if c["op"] == "norm":
        return {"bytes": M * K * e * (3 if c["add"] else 1) + 4 * K + codes, "flops": 8 * M * K}
    if c["op"] == "quantize":
        return {"bytes": M * K * e * (1 if c["act"] == "none" else 2) + codes, "flops": (4 if c["act"] == "none" else 12) * M * K}
    if c["op"] == "norm_grad":
        return {"bytes": M * K * e * (4 if c["add"] else 3) + 8 * K, "flops": 12 * M * K}
    if c["op"] == "gated_grad":
        return {"bytes": 5 * M * K * e, "flops": 16 * M * K}
    if c["op"] == "linear":
        return {"bytes": M * K + N * K + 4 * M + 4 * N * (2 if c["add"] else 1) + M * N * e, "flops": 2 * M * N * K}
    return {"bytes": M * N * e + N * K + 4 * N + M * K * e, "flops": 2 * M * N * K}


# ---------------------------------------------------------------- the definition in 64 bits
def _r32(v):
    """The definition's float32 results."""
    return v.float().double()


def _exact_values(v):
    """Of float32 rows held in 64 bits."""
    top = v.abs().max(1, keepdim=True).values
    s = _r32(top / 127)
    s[s == 0] = 1
    n = torch.round(_r32(v / s))
    return torch.minimum(torch.maximum(n, torch.full_like(n, -127)), torch.full_like(n, 127)) * s, s[:, 0]


def _exact_act(name, v):
    if name == "silu":
        e = torch.sigmoid(v)
        return v * e, e + v * e * torch.sigmoid(-v)
    c0 = math.sqrt(2 / math.pi)
    y = c0 * v * (1 + 0.044715 * v ** 2)
    t = torch.tanh(y)
    return v * (1 + t) / 2, (1 + t) / 2 + v / 2 / torch.cosh(y.clamp(-300, 300)) ** 2 * c0 * (1 + 3 * 0.044715 * v ** 2)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    K = c["K"]
    if c["op"] == "norm":
        h = s.x.double()
        if c["add"]:
            # float32 sums of two numbers of the type, then the type's rounding
            h = _r32(h + s.r.double()).to(s.x.dtype).double()
        rho = _r32((torch.linalg.vector_norm(h, dim=1) ** 2 / K + EPS) ** -0.5)
        out, scale = _exact_values(_r32(_r32(h * rho[:, None]) * s.w.double()))
        return [out, scale] + ([h] if c["add"] else [])
    if c["op"] == "quantize":
        v = s.x.double()
        if s.gate is not None:
            v = _r32(v * _exact_act(c["act"], s.gate.double())[0])
        return list(_exact_values(v))
    if c["op"] == "norm_grad":
        h, g = s.h.double(), s.dy.double()
        rho = (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / K + EPS) ** -0.5
        along = ((g * s.w.double()) * h).sum(1, keepdim=True)
        dx = g * s.w.double() * rho - h * along * rho ** 3 / K
        if c["add"]:
            dx += s.dh.double()
        return [dx, torch.einsum("mk,mk,m->k", g, h, rho[:, 0])]
    if c["op"] == "gated_grad":
        a, d = _exact_act(c["act"], s.gate.double())
        return [s.dh.double() * a, s.dh.double() * d * s.x.double()]
    if c["op"] == "linear":
        y = torch.matmul(s.x.double(), s.w.double().t().contiguous()) * torch.outer(s.xs.double(), s.ws.double())
        return [y + s.b.double() if c["add"] else y]
    return [torch.matmul(s.dy.double(), s.w.double() * s.ws.double()[:, None])]
