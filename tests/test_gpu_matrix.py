"""The matrix operators against plain 64-bit implementations of their definitions.

Tolerances, fixed before the first run:
  orthogonalisation  its products take operands rounded to 16-bit floating point, u = 2^-11.  A step rounds three operands
      (X, its Gram matrix off the diagonal, the polynomial off the diagonal); where a singular value grows, an earlier
      error grows with it and stays as large relative to it, near 1 the step contracts.  15 independent roundings of
      relative size u / sqrt(3) at most, times a gain of up to 1.5 from the polynomial: 1.6e-3.  Taken: 4 u = 2e-3 in the
      relative 2-norm, and 2^-8 more for a bfloat16 result.
  update             momentum: one rounding of the exact value, 2^-23 of the largest term.  Weights: three roundings of
      binary32 values plus eta scale times 4 u of the orthogonal factor's norm.
  codes              exact.
  products on codes  the integer sums are exact, so a binary32 result has at most the rounding of the sum to binary32 and
      two products: 4 x 2^-24 of its value; a bfloat16 result 2^-8.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U16 = 2.0 ** -11
A, B, C = 3.4445, -4.7750, 2.0315


@pytest.fixture(scope="module")
def rt():
    import paper_2005_10761_b200 as pkg
    from paper_2005_10761_b200 import build
    build.build()
    return pkg


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def orth64(u, steps=5, eps=1e-7, coef=None):
    x = u.double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for i in range(steps):
        a, b, c = coef[i] if coef else (A, B, C)
        if x.shape[-2] <= x.shape[-1]:
            g = x @ x.mT
            x = a * x + (b * g + c * (g @ g)) @ x
        else:
            g = x.mT @ x
            x = a * x + x @ (b * g + c * (g @ g))
    return x


def rel(x, y):
    return float((x.double() - y).norm() / y.norm())


def matrices(kind, batch, m, n, seed=0):
    g = gen(seed)
    noise = torch.randn((batch, m, n), generator=g, device="cuda")
    if kind == "gauss":
        return noise
    r = max(1, min(m, n) // 8)
    if kind == "low":
        return torch.randn((batch, m, r), generator=g, device="cuda") @ torch.randn((batch, r, n), generator=g, device="cuda") / r ** 0.5 + 0.1 * noise
    if kind == "sparse":
        return noise * (torch.rand((batch, m, n), generator=g, device="cuda") < 0.05) * torch.exp(torch.rand((batch, m, n), generator=g, device="cuda"))
    raise AssertionError(kind)


SHAPES = [(1, 64, 64), (1, 1, 1), (1, 1, 300), (2, 300, 1), (3, 2, 7), (1, 127, 129), (2, 129, 127), (5, 33, 65), (1, 128, 1000), (1, 1000, 130),
          (2, 257, 515), (1, 515, 1029), (1, 1029, 515), (1, 640, 640), (1, 1500, 2000), (1, 2000, 1500), (130, 20, 24)]


@pytest.mark.parametrize("batch,m,n", SHAPES)
@pytest.mark.parametrize("kind", ["gauss", "low", "sparse"])
def test_orthogonalize(rt, batch, m, n, kind):
    u = matrices(kind, batch, m, n) * 1e-3
    u[:, 0, 0] += 1e-3                      # no zero matrix among the sparse ones
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(batch, m, n))
    for src in (u, u.bfloat16()):
        want = orth64(src)
        for ty, tol in ((torch.float32, 4 * U16), (torch.bfloat16, 4 * U16 + 2.0 ** -8)):
            out = torch.full((batch, m, n), 7.0, dtype=ty, device="cuda")
            ctx.orthogonalize(src, out)
            ctx.poll_status()
            for z in range(batch):
                assert rel(out[z], want[z]) <= tol, (z, ty)
    ctx.close()


def test_orthogonalize_moves_singular_values_to_one(rt):
    u = matrices("gauss", 1, 384, 1024)
    out = torch.empty_like(u)
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(1, 384, 1024))
    ctx.orthogonalize(u, out)
    s = torch.linalg.svdvals(out[0].double())
    # the quintic's fixed interval around 1, widened by the operator's error in the 2-norm
    assert s.min() > 0.65 and s.max() < 1.25
    # the singular vectors stay: O^T U is symmetric positive
    p = out[0].double() @ u[0].double().T
    assert float((p - p.T).norm() / p.norm()) < 4 * U16 * 4


def test_orthogonalize_strides_batches_and_in_place(rt):
    m, n = 70, 150
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(4, n, n))
    base = matrices("gauss", 4, 91, 163, 3)
    src = base[:, 5:5 + m, 3:3 + n]                 # rows and matrices apart, odd offset
    out = torch.full((4, 80, 177), 9.0, dtype=torch.bfloat16, device="cuda")
    view = out[:, 1:1 + m, 7:7 + n]
    ctx.orthogonalize(src, view)
    want = orth64(src)
    assert rel(view, want) <= 4 * U16 + 2.0 ** -8
    untouched = out.clone()
    untouched[:, 1:1 + m, 7:7 + n] = 9.0
    assert bool((untouched == 9.0).all())
    same = src.bfloat16().contiguous()
    want = orth64(same)
    ctx.orthogonalize(same, same)
    assert rel(same, want) <= 4 * U16 + 2.0 ** -8
    one = src[2]
    o1 = torch.empty((m, n), device="cuda")
    ctx.orthogonalize(one, o1)
    assert rel(o1, orth64(one)) <= 4 * U16
    ctx.close()


def test_orthogonalize_empty_and_broken_matrices_stay_apart(rt):
    u = matrices("gauss", 5, 40, 96)
    u[1] = 0.0
    u[2, 3, 4] = float("nan")
    u[3, 0, 0] = float("inf")
    u[4] *= 1e-30                                      # squares below the binary32 range
    out = torch.full_like(u, 5.0)
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(5, 40, 96))
    ctx.orthogonalize(u, out, eps=0.0)
    assert rel(out[0], orth64(u[0], eps=0.0)) <= 4 * U16
    assert bool((out[1] == 0).all())
    assert bool(out[2].isnan().all()) and bool(out[3].isnan().any())
    assert rel(out[4], orth64(u[4], eps=0.0)) <= 4 * U16
    big = matrices("gauss", 1, 40, 96, 8) * 1e30       # squares above it
    ctx.orthogonalize(big, out[:1])
    assert rel(out[0], orth64(big[0])) <= 4 * U16
    ctx.close()


@pytest.mark.parametrize("steps", [1, 3, 8])
def test_orthogonalize_steps_and_coefficients(rt, steps):
    u = matrices("low", 1, 200, 333, 4)
    out = torch.empty_like(u)
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(1, 200, 333))
    ctx.orthogonalize(u, out, steps=steps)
    assert rel(out, orth64(u, steps)) <= 4 * U16 * max(1.0, math.sqrt(steps / 5))
    coef = [(1.5 + 0.1 * i, -0.5, 0.01 * i) for i in range(steps)]       # the cubic step, nearly
    ctx.orthogonalize(u, out, steps=steps, coef=coef)
    assert rel(out, orth64(u, steps, coef=coef)) <= 4 * U16 * max(1.0, math.sqrt(steps / 5))
    ctx.close()


@pytest.mark.parametrize("batch,m,n", [(1, 64, 64), (2, 300, 70), (4, 129, 260), (1, 1, 9), (1, 700, 1500)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_orthogonal_update(rt, batch, m, n, nesterov):
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(batch, m, n))
    g = matrices("sparse", batch, m, n, 1) * 1e-3
    v = matrices("low", batch, m, n, 2) * 1e-3
    w = matrices("gauss", batch, m, n, 3) * 0.05
    wide = torch.zeros((batch, m, n + 5), device="cuda")
    wide[..., 2:2 + n] = w
    weights = wide[..., 2:2 + n]
    eta, mu, decay, scale = 0.02, 0.9, 0.1, 0.2 * max(m, n) ** 0.5
    v64 = mu_exact(mu) * v.double() + g.double()
    for _ in range(2):                     # twice: the state carries over
        want_v = v64
        ctx.orthogonal_update(g, v, weights, eta, mu, nesterov=nesterov, decay=decay, scale=scale)
        ctx.poll_status()
        big = (want_v.abs() + g.abs().double()).max()
        assert float((v.double() - want_v).abs().max() / big) <= 2.0 ** -23
        u = g.double() + mu_exact(mu) * v.double() if nesterov else v.double()
        o = orth64(u)
        want_w = w.double() * (1 - eta * decay) - eta * scale * o
        for z in range(batch):
            err = float((weights[z].double() - want_w[z]).norm())
            assert err <= 3 * 2.0 ** -24 * float(want_w[z].norm()) + eta * scale * 4 * U16 * float(o[z].norm())
        w = weights.clone()
        v64 = mu_exact(mu) * v.double() + g.double()
    assert bool((wide[..., :2] == 0).all()) and bool((wide[..., 2 + n:] == 0).all())
    ctx.close()


def mu_exact(mu):
    return float(torch.tensor(mu, dtype=torch.float32).double())


# ------------------------------------------------------------------------------------------------ codes

def code64(v, dim):
    """By definition: scale and quotient rounded to binary32."""
    v = v.float()
    top = v.abs().amax(dim, keepdim=True)
    s = (top.double() / 127).float()
    q = (v.double() / s.double()).float().double().round().clamp(-127, 127)
    s = torch.where(top.isfinite(), s, torch.full_like(s, float("nan")))
    return torch.where(s > 0, q, torch.zeros_like(q)), s.double()


def near(got, want, ty):
    tol = 4 * 2.0 ** -24 if ty == torch.float32 else 2.0 ** -8
    d = (got.double() - want).abs()
    bad = ~(d <= tol * want.abs() + 1e-300)
    assert bool((got.isnan() == want.isnan()).all())
    assert not bool((bad & ~want.isnan()).any()), (float(d.max()), int(bad.sum()))


def tokens_of(t, k, seed, ty):
    g = gen(seed)
    x = torch.randn((t, k), generator=g, device="cuda") * torch.exp(torch.randn((t, 1), generator=g, device="cuda"))
    return x.to(ty)


@pytest.mark.parametrize("n_out,n_in", [(1, 1), (3, 16), (64, 64), (127, 130), (129, 1500), (1000, 257), (300, 5000)])
@pytest.mark.parametrize("ty", [torch.float32, torch.bfloat16])
def test_code_weights(rt, n_out, n_in, ty):
    w = tokens_of(n_out, n_in, 5, ty)
    if n_out > 2:
        w[1] = 0.0
        w[2] *= 1e-38                                   # scales among the subnormal numbers
    ctx = rt.MatrixContext(0)
    coded = rt.CodedWeights(n_out, n_in)
    ctx.code_weights(w, coded)
    q, s = code64(w, 1)
    assert torch.equal(coded.scales.double(), s.flatten())
    assert torch.equal(coded.codes[:, :n_in].double(), q)
    assert torch.equal(coded.codes_t[:, :n_out].t().double(), q)
    assert torch.equal(coded.dense().double(), (q * s).float().double())
    flat = rt.CodedWeights(n_out, n_in, transposed=False)
    ctx.code_weights(w, flat)
    assert torch.equal(flat.codes, coded.codes) and flat.codes_t is None
    ctx.close()


PRODUCTS = [(1, 1, 1), (1, 1500, 6000), (1, 8192, 40), (2, 130, 257), (3, 16, 127), (4, 4100, 300), (5, 1000, 1000), (7, 127, 129), (8, 1500, 700),
            (9, 2048, 512), (16, 640, 384), (17, 129, 128), (24, 4096, 1000), (31, 33, 65), (33, 1500, 300), (48, 500, 2100), (64, 256, 256), (65, 1024, 640),
            (100, 2000, 130), (129, 128, 1), (200, 1, 200), (300, 700, 515), (700, 1500, 1000), (1025, 384, 900)]


@pytest.mark.parametrize("tokens,n_in,n_out", PRODUCTS)
@pytest.mark.parametrize("ty", [torch.float32, torch.bfloat16])
def test_coded_product(rt, tokens, n_in, n_out, ty):
    ctx = rt.MatrixContext(rt.coded_scratch(tokens, n_out, n_in))
    w, x = tokens_of(n_out, n_in, 1, torch.float32) * 0.05, tokens_of(tokens, n_in, 2, ty)
    if tokens > 2:
        x[1] = 0.0
    coded = rt.CodedWeights(n_out, n_in)
    ctx.code_weights(w, coded)
    out = torch.full((tokens, n_out), 3.0, dtype=ty, device="cuda")
    ctx.coded_product(x, coded, out)
    ctx.poll_status()
    qx, sx = code64(x, 1)
    qw, sw = code64(w, 1)
    near(out, (qx @ qw.t()) * sx * sw.t(), ty)
    # rows apart and at odd offsets
    xs = torch.zeros((tokens, n_in + 3), dtype=ty, device="cuda")
    xs[:, 1:1 + n_in] = x
    outs = torch.full((tokens, n_out + 5), 3.0, dtype=ty, device="cuda")
    ctx.coded_product(xs[:, 1:1 + n_in], coded, outs[:, 3:3 + n_out])
    assert torch.equal(outs[:, 3:3 + n_out], out)
    outs[:, 3:3 + n_out] = 3.0
    assert bool((outs == 3.0).all())
    ctx.close()


@pytest.mark.parametrize("tokens", [1, 5, 40, 300])
def test_coded_product_of_broken_rows(rt, tokens):
    """A token or a channel with an infinity or a NaN is NaN throughout, and nothing else is."""
    n_in, n_out = 200, 300
    ctx = rt.MatrixContext(rt.coded_scratch(tokens, n_out, n_in))
    w, x = tokens_of(n_out, n_in, 1, torch.float32), tokens_of(tokens, n_in, 2, torch.float32)
    w[7, 3] = float("inf")
    w[9, 0] = float("nan")
    if tokens > 1:
        x[0, 5] = float("-inf")
        x[tokens - 1, 199] = float("nan")
    coded = rt.CodedWeights(n_out, n_in)
    ctx.code_weights(w, coded)
    out = torch.zeros((tokens, n_out), device="cuda")
    ctx.coded_product(x, coded, out)
    qx, sx = code64(x, 1)
    qw, sw = code64(w, 1)
    want = (qx @ qw.t()) * sx * sw.t()
    assert bool(want[:, 7].isnan().all()) and not bool(want[tokens // 2, 8:9].isnan().any())
    near(out, want, torch.float32)
    ctx.close()


GRADS = [(1, 1, 1), (1, 300, 200), (2, 16, 16), (7, 127, 129), (64, 640, 384), (65, 129, 700), (127, 1500, 300), (300, 257, 515), (700, 1500, 600), (1025, 384, 130)]


@pytest.mark.parametrize("tokens,n_in,n_out", GRADS)
@pytest.mark.parametrize("ty,wty", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_coded_gradients(rt, tokens, n_in, n_out, ty, wty):
    ctx = rt.MatrixContext(rt.coded_scratch(tokens, n_out, n_in))
    w, x = tokens_of(n_out, n_in, 1, torch.float32) * 0.05, tokens_of(tokens, n_in, 2, ty)
    dy = tokens_of(tokens, n_out, 3, ty) * 1e-3
    if tokens > 2:
        dy[1] = 0.0
        x[:, 0] = 0.0
    coded = rt.CodedWeights(n_out, n_in)
    ctx.code_weights(w, coded)
    dx = torch.full((tokens, n_in), 3.0, dtype=ty, device="cuda")
    dw = torch.full((n_out, n_in + 7), 3.0, dtype=wty, device="cuda")
    ctx.coded_gradients(dy, x, coded, dx, dw[:, 2:2 + n_in])
    ctx.poll_status()
    qw, sw = code64(w, 1)
    q, s = code64(dy.float() * sw.float().t(), 1)
    near(dx, (q @ qw) * s, ty)
    qy, sy = code64(dy, 0)
    qx, sx = code64(x, 0)
    near(dw[:, 2:2 + n_in], (qy.t() @ qx) * sy.t() * sx, wty)
    assert bool((dw[:, :2] == 3.0).all()) and bool((dw[:, 2 + n_in:] == 3.0).all())
    # each alone gives the same
    dx2, dw2 = torch.zeros_like(dx), torch.zeros((n_out, n_in), dtype=wty, device="cuda")
    ctx.coded_gradients(dy, None, coded, dx=dx2)
    ctx.coded_gradients(dy, x, coded, dw=dw2)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw[:, 2:2 + n_in])
    ctx.close()


def test_coded_gradients_against_differences(rt):
    """Along random directions, the gradients agree with central differences of sum(dy * x W^T) in 64 bits up to the
    rounding to codes: a code's error is uniform over one step of max / 127 <= 6 rms / 127, 1.4 % of the rms for each of
    the two factors, 2 % of the gradient's norm together; 3 % taken."""
    t, k, n = 256, 300, 200
    ctx = rt.MatrixContext(rt.coded_scratch(t, n, k))
    g = gen(11)
    w, x, dy = (torch.randn(s, generator=g, device="cuda") for s in ((n, k), (t, k), (t, n)))
    coded = rt.CodedWeights(n, k)
    ctx.code_weights(w, coded)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ctx.coded_gradients(dy, x, coded, dx, dw)
    f = lambda xx, ww: float((dy.double() * (xx @ ww.t())).sum())       # noqa: E731
    X, W = x.double(), w.double()
    for which, grad, at in (("x", dx, X), ("w", dw, W)):
        for i in range(4):
            # a direction with a part along the gradient, so that the difference is not noise alone
            d = torch.randn(at.shape, generator=g, device="cuda", dtype=torch.float64)
            d = d / d.norm() + (dy.double() @ W if which == "x" else dy.double().t() @ X) / (dy.double() @ W if which == "x" else dy.double().t() @ X).norm()
            h = 1e-3
            diff = (f(X + h * d, W) - f(X - h * d, W)) / (2 * h) if which == "x" else (f(X, W + h * d) - f(X, W - h * d)) / (2 * h)
            got = float((grad.double() * d).sum())
            assert abs(got - diff) <= 0.03 * float(grad.double().norm() * d.norm())
    ctx.close()


def test_no_tokens(rt):
    ctx = rt.MatrixContext(rt.coded_scratch(0, 40, 30))
    coded = rt.CodedWeights(40, 30)
    ctx.code_weights(torch.ones((40, 30), device="cuda"), coded)
    none_x, none_y = torch.empty((0, 30), device="cuda"), torch.empty((0, 40), device="cuda")
    ctx.coded_product(none_x, coded, none_y)
    dw = torch.full((40, 33), 2.0, device="cuda")
    ctx.coded_gradients(none_y, none_x, coded, torch.empty_like(none_x), dw[:, :30])
    assert bool((dw[:, :30] == 0).all()) and bool((dw[:, 30:] == 2.0).all())
    ctx.close()


def test_largest_sums_are_exact(rt):
    """All codes at +-127 over the longest supported contraction: the sum is 127 * 127 * 131072 = 2114060288 < 2^31."""
    k = 131072
    ctx = rt.MatrixContext(rt.coded_scratch(40, 3, k))
    coded = rt.CodedWeights(3, k, transposed=False)
    w = torch.ones((3, k), device="cuda")
    w[1] = -1.0
    w[2, 1::2] = -1.0
    ctx.code_weights(w, coded)
    for t in (1, 5, 40):
        out = torch.zeros((t, 3), device="cuda")
        ctx.coded_product(torch.ones((t, k), device="cuda"), coded, out)
        near(out, torch.tensor([1.0, -1.0, 0.0], device="cuda", dtype=torch.float64).expand(t, 3) * (2114060288.0 * float(coded.scales[0].double()) ** 2), torch.float32)
    with pytest.raises(rt.RTopKError) as e:
        big = rt.MatrixContext(rt.coded_scratch(1, 1, k + 16))
        c = rt.CodedWeights(1, k + 16, transposed=False)
        big.coded_product(torch.ones((1, k + 16), device="cuda"), c, torch.zeros((1, 1), device="cuda"))
    assert e.value.status == 4
    ctx.close()


# ------------------------------------------------------------------------------------------------ calls

def test_same_result_on_another_stream_in_a_graph_and_every_time(rt):
    m, n, t = 200, 390, 70
    ctx = rt.MatrixContext(max(rt.orthogonalize_scratch(2, m, n), rt.coded_scratch(t, n, m)))
    u, x, dy = matrices("gauss", 2, m, n), tokens_of(t, m, 1, torch.bfloat16), tokens_of(t, n, 2, torch.bfloat16)
    coded = rt.CodedWeights(n, m)
    ctx.code_weights(tokens_of(n, m, 3, torch.float32), coded)

    def all_of():
        o, y = torch.empty((2, m, n), dtype=torch.bfloat16, device="cuda"), torch.empty((t, n), dtype=torch.bfloat16, device="cuda")
        dx, dw = torch.empty_like(x), torch.empty((n, m), device="cuda")

        def call():
            ctx.orthogonalize(u, o)
            ctx.coded_product(x, coded, y)
            ctx.coded_gradients(dy, x, coded, dx, dw)
        return (o, y, dx, dw), call

    first, call = all_of()
    call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        again, call = all_of()
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    replayed, call = all_of()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(2):
        for r in replayed:
            r.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, replayed))
    ctx.poll_status()
    assert ctx.launch_count() > 0
    ctx.close()


def test_refusals(rt):
    f = lambda *s: torch.zeros(s, device="cuda")       # noqa: E731
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(1, 32, 64))

    def status(call):
        with pytest.raises(rt.RTopKError) as e:
            call()
        return e.value.status

    u, o = f(32, 64), f(32, 64)
    assert status(lambda: ctx.orthogonalize(u, o, steps=0)) == 1
    assert status(lambda: ctx.orthogonalize(u, o, steps=65)) == 1
    assert status(lambda: ctx.orthogonalize(u, o, eps=-1.0)) == 1
    assert status(lambda: ctx.orthogonalize(u, o, eps=float("nan"))) == 1
    assert status(lambda: ctx.orthogonalize(u, o, steps=1, coef=[(1.0, float("inf"), 0.0)])) == 1
    assert status(lambda: ctx.orthogonalize(f(320, 640), f(320, 640))) == 1            # more scratch than there is
    for bad in (dict(eta=-1.0), dict(eta=float("nan")), dict(mu=1.0), dict(mu=-0.1), dict(decay=-1.0), dict(scale=float("inf"))):
        assert status(lambda: ctx.orthogonal_update(u, f(32, 64), o, **{**dict(eta=0.1, mu=0.9), **bad})) == 1
    for call in (lambda: ctx.orthogonalize(u, f(32, 63)), lambda: ctx.orthogonalize(f(64, 32).t(), o), lambda: ctx.orthogonalize(f(4), f(4)),
                 lambda: ctx.orthogonalize(u, o, coef=[(1.0, 0.0, 0.0)])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        ctx.orthogonalize(u.half(), o)
    with pytest.raises(TypeError):
        ctx.orthogonal_update(u.bfloat16(), f(32, 64), o, 0.1, 0.9)
    coded = rt.CodedWeights(40, 30)
    small = rt.MatrixContext(0)
    assert status(lambda: small.coded_product(f(300, 30), coded, f(300, 40))) == 1
    with pytest.raises(TypeError):
        ctx.coded_product(f(3, 30), coded, f(3, 40).bfloat16())
    with pytest.raises(ValueError):
        ctx.coded_product(f(3, 31), coded, f(3, 40))
    with pytest.raises(ValueError):
        ctx.coded_gradients(f(3, 40), f(3, 30), rt.CodedWeights(40, 30, transposed=False), f(3, 30), f(40, 30))
    assert status(lambda: ctx.coded_gradients(f(3, 40), f(3, 30), coded)) == 1
    lib, p = rt.load_library(), coded.codes.data_ptr()
    x, y = f(3, 30), f(3, 40)
    ok = (ctx._h, x.data_ptr(), 0, 30, p, 128, coded.scales.data_ptr(), 3, 40, 30, y.data_ptr(), 40, None)
    for at, v in ((0, None), (1, None), (2, 2), (3, 29), (4, None), (4, p + 8), (5, 24), (5, 120), (6, None), (7, -1), (8, 0), (9, 0), (10, None), (11, 39)):
        args = list(ok)
        args[at] = v
        assert lib.rtopk_coded_product(*args) == 1, (at, v)
    with pytest.raises(rt.RTopKError):
        rt.orthogonalize_scratch(0, 3, 3)
    with pytest.raises(rt.RTopKError):
        rt.coded_scratch(-1, 3, 3)
    with pytest.raises(rt.RTopKError):
        rt.MatrixContext(-1)
    torch.cuda.synchronize()
    ctx.close()
    small.close()
