"""The matrix operators of a training round: the cases they are timed and checked on.

Four operators around the sparsified exchange of Algorithm 1:

  orth     the orthogonal factor of a matrix by five Newton-Schulz steps,
               X <- U / (||U||_F + eps);  X <- a X + b (X X^T) X + c (X X^T)^2 X, five times;
  update   the master update of a weight matrix with it: v <- mu v + g;  u = g + mu v;
               w <- (1 - eta lambda) w - eta s orth(u);
  product  a worker's linear layer on 8-bit codes: y = x W^T with W held as codes and one scale for
           each output channel (what the master broadcasts), x coded for each token inside the call;
  grads    the gradients of that layer, both products on 8-bit codes: with respect to x (the output's
           gradient, times the channel scales, coded for each token) and with respect to W (both factors
           coded for each channel over the tokens), the latter being the worker's gradient g.

A row (or column) v is coded as q = rint(v / s), clamped to +-127, with s = max|v| / 127, every step
rounded to binary32; an all-zero row has s = 0 and q = 0.

`own` chooses between the plain form in elementary torch operations and the library's calls.
"""
import math

import torch

own = False

A, B, C = 3.4445, -4.7750, 2.0315      # the coefficients of the quintic step
STEPS, EPS = 5, 1e-7

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the smallest call: one projection of a small head, where only latency counts
        {"name": "orth 64x64 f32", "op": "orth", "batch": 1, "m": 64, "n": 64, "type": "f32"},
        # a few odd-sized tall matrices of one shape in one call, bfloat16
        {"name": "orth 3x1029x515 bf16", "op": "orth", "batch": 3, "m": 1029, "n": 515, "type": "bf16"},
        # a square projection of a mid-sized model
        {"name": "orth 2048x2048 bf16", "op": "orth", "batch": 1, "m": 2048, "n": 2048, "type": "bf16"},
        # the output layer of the two-layer LSTM workload: very wide, rows that are no multiple of a tile
        {"name": "orth 1500x10000 f32", "op": "orth", "batch": 1, "m": 1500, "n": 10000, "type": "f32"},
        # the master update of the LSTM's four recurrent tensors in one call
        {"name": "update 4x6000x1500", "op": "update", "batch": 4, "m": 6000, "n": 1500, "eta": 2e-4, "mu": 0.95, "decay": 0.1},
        # the master update of one small square projection
        {"name": "update 512x512", "op": "update", "batch": 1, "m": 512, "n": 512, "eta": 2e-4, "mu": 0.9, "decay": 0.0},
        # one token through the LSTM's gates: reading the codes is all the work
        {"name": "product 1x1500->6000 bf16", "op": "product", "tokens": 1, "n_in": 1500, "n_out": 6000, "type": "bf16"},
        # a small batch of sequences, one token each, through a large layer
        {"name": "product 24x8192->8192 bf16", "op": "product", "tokens": 24, "n_in": 8192, "n_out": 8192, "type": "bf16"},
        # a training batch through the LSTM's output layer, binary32 activations
        {"name": "product 700x1500->10000 f32", "op": "product", "tokens": 700, "n_in": 1500, "n_out": 10000, "type": "f32"},
        # a long batch through a square layer: the tensor cores' case
        {"name": "product 8192x4096->8192 bf16", "op": "product", "tokens": 8192, "n_in": 4096, "n_out": 8192, "type": "bf16"},
        # the gradients of the LSTM's gates for a training batch
        {"name": "grads 700x1500->6000 f32", "op": "grads", "tokens": 700, "n_in": 1500, "n_out": 6000, "type": "f32"},
        # the gradients of a large layer for a long batch
        {"name": "grads 8192x4096->4096 bf16", "op": "grads", "tokens": 8192, "n_in": 4096, "n_out": 4096, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["orth", "update", "product", "grads"])
    if op in ("orth", "update"):
        m, n = _log(rng, 48, 6000), _log(rng, 48, 6000)
        if min(m, n) > 2048:
            m = 2048
        a, z = sorted((m, n))
        most = min(4e11 / (3.0 * a * a * z + (4 * STEPS - 3) * a ** 3), 3.5e7 / (a * z))
        case = {"op": op, "batch": min(_log(rng, 1, 8), max(1, int(most))), "m": m, "n": n}
        if op == "orth":
            case["type"] = rng.choice(["f32", "bf16"])
        else:
            case.update(eta=2e-4, mu=rng.choice([0.9, 0.95]), decay=rng.choice([0.0, 0.1]))
        return case
    tokens = _log(rng, 1, 8192) if op == "product" else _log(rng, 64, 8192)
    return {"op": op, "tokens": tokens, "n_in": _log(rng, 256, 4096), "n_out": _log(rng, 256, 4096), "type": rng.choice(["f32", "bf16"])}


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _matrices(batch, m, n, gen):
    """What a matrix of accumulated gradients looks like: a decaying spectrum over an eighth of the directions, a skew over
    the rows, and noise."""
    r = max(1, min(m, n) // 8)
    s = torch.arange(1, r + 1, device="cuda", dtype=torch.float32).rsqrt()
    g = (_normal((batch, m, r), gen) * s) @ _normal((batch, r, n), gen) / s.square().sum().sqrt()
    return (g * torch.exp(0.5 * _normal((batch, m, 1), gen)) + 0.3 * _normal((batch, m, n), gen)) * 1e-3


def _tokens(shape, gen):
    """Activations and their gradients: normal, a skew over the tokens, and a few channels that stand out."""
    x = _normal(shape, gen) * torch.exp(0.5 * _normal((shape[0], 1), gen))
    return x * (1 + 7 * (torch.rand((1, shape[1]), generator=gen, device="cuda") < 0.01))


def _code(v, dim):
    """The codes of v along `dim` as binary32 numbers, and their scales."""
    v = v.float()
    s = v.abs().amax(dim, keepdim=True)
    s = s / torch.full_like(s, 127)      # torch turns a division by a number into a product with its reciprocal
    return torch.where(s > 0, (v / s).round().clamp(-127, 127), torch.zeros_like(v)), s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] in ("orth", "update"):
        b, m, n = case["batch"], case["m"], case["n"]
        if case["op"] == "orth":
            s["u"] = _matrices(b, m, n, gen).to(TYPES[case["type"]])
            s["out"] = torch.empty((b, m, n), dtype=torch.bfloat16, device="cuda")
        else:
            s["v"] = _matrices(b, m, n, gen)
            # the average of sparse messages: one coordinate in a hundred
            s["g"] = _normal((b, m, n), gen) * 2e-3 * (torch.rand((b, m, n), generator=gen, device="cuda") < 0.01)
            s["w"] = _normal((b, m, n), gen) * 0.05
            s["scale"] = 0.2 * math.sqrt(max(m, n))
        if own:
            import paper_2005_10761_b200 as rt
            s["ctx"] = rt.MatrixContext(rt.orthogonalize_scratch(b, m, n))
        return s
    t, k, n, ty = case["tokens"], case["n_in"], case["n_out"], TYPES[case["type"]]
    s["x"] = _tokens((t, k), gen).to(ty)
    w = _normal((n, k), gen) * (0.05 * torch.exp(0.3 * _normal((n, 1), gen)))
    s["codes"], s["scales"] = _code(w, 1)
    if case["op"] == "product":
        s["y"] = torch.empty((t, n), dtype=ty, device="cuda")
    else:
        s["dy"] = (_tokens((t, n), gen) * 1e-3).to(ty)
        s["dx"] = torch.empty((t, k), dtype=ty, device="cuda")
        s["dw"] = torch.empty((n, k), dtype=ty, device="cuda")
    if own:
        import paper_2005_10761_b200 as rt
        s["ctx"] = rt.MatrixContext(rt.coded_scratch(t, n, k))
        s["coded"] = rt.CodedWeights(n, k)
        s["ctx"].code_weights(w, s["coded"])
    return s


def _orth(u):
    x = u.float()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    for _ in range(STEPS):
        g = x @ x.transpose(1, 2)
        x = A * x + (B * g + C * (g @ g)) @ x
    return x.transpose(1, 2) if tall else x


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        ctx = state["ctx"]
        if op == "orth":
            ctx.orthogonalize(state["u"], state["out"])
            return state["out"]
        if op == "update":
            ctx.orthogonal_update(state["g"], state["v"], state["w"], case["eta"], case["mu"], decay=case["decay"], scale=state["scale"])
            return state["v"], state["w"]
        if op == "product":
            ctx.coded_product(state["x"], state["coded"], state["y"])
            return state["y"]
        ctx.coded_gradients(state["dy"], state["x"], state["coded"], state["dx"], state["dw"])
        return state["dx"], state["dw"]
    if op == "orth":
        state["out"].copy_(_orth(state["u"]))
        return state["out"]
    if op == "update":
        g, v, w = state["g"], state["v"], state["w"]
        v.mul_(case["mu"]).add_(g)
        o = _orth(g + case["mu"] * v)
        w.mul_(1 - case["eta"] * case["decay"]).sub_(o, alpha=case["eta"] * state["scale"])
        return v, w
    codes, scales, x = state["codes"], state["scales"], state["x"]
    if op == "product":
        q, s = _code(x, 1)
        state["y"].copy_((q @ codes.t()) * s * scales.t())
        return state["y"]
    dy = state["dy"]
    q, s = _code(dy.float() * scales.t(), 1)
    state["dx"].copy_((q @ codes) * s)
    qy, sy = _code(dy, 0)
    qx, sx = _code(x, 0)
    state["dw"].copy_((qy.t() @ qx) * sy.t() * sx)
    return state["dx"], state["dw"]


def work(case):
    if case["op"] in ("orth", "update"):
        b, m, n = case["batch"], *sorted((case["m"], case["n"]))
        # The steps commute, so that one Gram product, 4 * STEPS - 3 products of symmetric m x m matrices and one
        # product with X do; each symmetric product needs half of its entries.
        flops = b * (3.0 * m * m * n + (4 * STEPS - 3) * m ** 3)
        size = {"f32": 4, "bf16": 2}[case["type"]] + 2 if case["op"] == "orth" else 5 * 4
        return {"bytes": b * m * n * size, "flops": flops}
    t, k, n = case["tokens"], case["n_in"], case["n_out"]
    e = 4 if case["type"] == "f32" else 2
    if case["op"] == "product":
        return {"bytes": e * t * (k + n) + n * k + 4 * n, "flops": 2.0 * t * k * n}
    return {"bytes": e * (2 * t * k + t * n + n * k) + n * k + 4 * n, "flops": 4.0 * t * k * n}


def _orth64(u):
    """By the right side: X (a + b G + c G^2) with G = X^T X over the shorter side's transpose."""
    x = u.double()
    if x.shape[1] < x.shape[2]:
        return _orth64(u.transpose(1, 2)).transpose(1, 2)
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + EPS)
    one = torch.eye(x.shape[2], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        g = torch.bmm(x.transpose(1, 2), x)
        x = torch.bmm(x, A * one + torch.bmm(g, B * one + C * g))
    return x


def _code64(v, dim):
    """Scale and quotient are rounded to binary32 by definition; everything else is exact."""
    s = (v.abs().max(dim, keepdim=True).values.double() / 127).float()
    q = (v.double() / s.double()).float().double()
    q = torch.where(s == 0, torch.zeros_like(q), torch.round(q))
    return q.clamp(-127, 127), s.double()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "orth":
        return _orth64(s["u"])
    if op == "update":
        g, v, mu = s["g"].double(), s["v"].double(), case["mu"]
        v = mu * v + g
        w = s["w"].double() * (1 - case["eta"] * case["decay"]) - case["eta"] * s["scale"] * _orth64(g + mu * v)
        return v, w
    codes, scales, x = s["codes"].double(), s["scales"].double().flatten(), s["x"].float()
    if op == "product":
        q, sx = _code64(x, 1)
        return torch.einsum("tk,nk->tn", q * sx, codes * scales[:, None])
    dy = s["dy"].float()
    q, sd = _code64(dy * s["scales"].flatten(), 1)
    dx = torch.einsum("tn,nk->tk", q * sd, codes)
    qy, sy = _code64(dy, 0)
    qx, sx = _code64(x, 0)
    return dx, torch.einsum("tn,tk->nk", qy * sy, qx * sx)
