"""A worker's layers against plain 64-bit implementations of their definitions: 4-bit codes, their products and gradients, dropout,
layer normalisation and its gradients.

Tolerances, fixed before the first run (u = 2^-24, half a step of binary32; a bfloat16 result adds 2^-8 of its value):
  codes and masks   exact.
  products on codes   the 64 products of an instruction are exact; the tensor core drops what falls below the last bit of its accumulator,
      taken as 2^-22 of the sum of the terms' magnitudes for each instruction, and up to eight parts are added with one rounding
      each: (K / 64 + 8) 2^-22 sum |x| |w|.
  normalisation   t: two roundings; a row's sums pass through at most 8 + 31 + 5 + 16 = 60 additions (columns of a thread, pieces beyond
      them, lanes, warps), so mean and differences are within 64 u of the row's largest |t|, M; rows of more than 2^14 columns add cols / 4096.
      The variance moves by twice that over the standard deviation and by 64 u of itself.  With D = 64 u M rstd: h within D (1 + 2 |h|) + 64 u |h|.
  its gradients   h from given mean and rstd: three roundings, 4 u (|t| + |mean|) rstd; each row sum within 64 u of its terms' magnitudes.
  sums over rows   64 u of the terms' magnitudes for the additions in 32 bits (rows of a block in turn, then eight warps; more rows: rows / 4096 more).
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def rt():
    import paper_2005_10761_b200 as pkg
    from paper_2005_10761_b200 import build
    build.build()
    return pkg


def normal(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def rounding(ty, v):
    return (2.0 ** -8 if ty == torch.bfloat16 else U) * v.abs()


def close(got, want, tol, what=""):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got.double() - want).abs() - tol).nan_to_num().max()))


# ------------------------------------------------------------------------------------------------- definitions
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def coded(v, tile=1, dim=1):
    """The values of the 4-bit codes of a matrix, in 64 bits: blocks of 32 along dim, `tile` lines to a scale."""
    if dim == 0:
        return coded(v.t(), tile).t()
    v = v.double()
    m, n = v.shape
    pad = torch.nn.functional.pad(v, (0, -n % 32, 0, -m % tile))
    blocks = pad.view(-1, tile, pad.shape[1] // 32, 32)
    most = blocks.abs().amax((1, 3), keepdim=True)
    powers = torch.tensor([2.0 ** e for e in range(-127, 128)], dtype=torch.float64, device=v.device)
    step = powers[torch.searchsorted(6 * powers, most.nan_to_num(1.0, 1.0)).clamp(max=254)]
    table = VALUES.to(v.device)
    middle = (table[1:] + table[:-1]) / 2
    q = blocks.abs() / step
    low = torch.bucketize(q, middle).clamp(max=7)
    up = (low < 7) & (q == middle[low.clamp(max=6)]) & (low % 2 == 1)
    out = torch.sign(blocks) * table[low + up.long()] * step
    out = torch.where(most.isfinite(), out, torch.full_like(out, float("nan")))
    return out.reshape(pad.shape)[:m, :n]


def kept(rows, cols, p, seed, step=0, worker=0, site=0, row0=0):
    """(mask, factor) by Philox4x32-10, written with unsigned 64-bit products on the host."""
    u = np.uint64
    g = -(-cols // 8)
    c = [np.broadcast_to(np.arange(g, dtype=u), (rows, g)), np.broadcast_to(np.arange(row0, row0 + rows, dtype=u)[:, None], (rows, g)),
         np.full((rows, g), 2 ** 31 + 65536 * site + worker, dtype=u), np.full((rows, g), step, dtype=u)]
    for i in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        k0, k1 = u((seed + i * 0x9E3779B9) % 2 ** 32), u(((seed >> 32) + i * 0xBB67AE85) % 2 ** 32)
        c = [(b >> u(32)) ^ c[1] ^ k0, b & u(0xFFFFFFFF), (a >> u(32)) ^ c[3] ^ k1, a & u(0xFFFFFFFF)]
    numbers = np.stack(c, 2).astype(np.uint32).view(np.uint16).reshape(rows, 8 * g)[:, :cols]
    limit = min(round(65536 * p), 65535)
    return torch.from_numpy(numbers >= limit).cuda(), float(np.float32(65536 / (65536 - limit)))


# ------------------------------------------------------------------------------------------------- 4-bit codes
@pytest.mark.parametrize("n_out,n_in", [(1, 1), (1, 32), (3, 33), (31, 7), (32, 32), (33, 129), (128, 128), (130, 257), (257, 255), (500, 1500), (129, 1029), (1029, 640)])
@pytest.mark.parametrize("ty", TYPES)
def test_micro_weights(rt, n_out, n_in, ty):
    base = (normal(n_out + 2, n_in + 5) * torch.exp(normal(n_out + 2, 1, seed=1)) * 0.05).to(ty)
    base[0, 0] = 0.0
    ctx = rt.MatrixContext(0)
    for w in (base[:n_out, :n_in].contiguous(), base[1:1 + n_out, 3:3 + n_in]):
        for tile in (1, 32):
            m = rt.MicroWeights(n_out, n_in, transposed=tile == 32, tile=tile)
            for t in (m.codes, m.scales, m.codes_t, m.scales_t):
                if t is not None:
                    t.fill_(255)
            ctx.micro_weights(w, m)
            want = coded(w, tile)
            assert torch.equal(m.dense().double(), want)
            if tile == 32:
                t = rt.MicroWeights(n_in, n_out, transposed=False)
                t.codes, t.scales = m.codes_t, m.scales_t
                assert torch.equal(t.dense().double(), want.t())
    ctx.close()


def test_micro_codes_at_the_middles_and_the_ends_of_the_range(rt):
    """Every middle between two codes, both signs, in blocks whose scale the largest value fixes; then scales from the smallest numbers to the largest."""
    ctx = rt.MatrixContext(0)
    near = []
    for v in [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]:
        near += [v, -v, float(np.nextafter(np.float32(v), np.float32(9))), float(np.nextafter(np.float32(v), np.float32(0)))]
    row = torch.tensor((near + [6.0, -6.0, 0.0, -0.0])[:32], device="cuda")
    assert row.numel() == 32 and float(row.abs().max()) == 6.0
    powers = torch.tensor([2.0 ** e for e in range(-126, 125)], device="cuda")
    w = row * powers[:, None]
    w = torch.cat([w, row[:, None].expand(32, 32).t() * 2.0 ** -126 / 64,                         # subnormal
                   torch.tensor([[float(np.nextafter(np.float32(6), np.float32(9)))] + [1.0] * 31], device="cuda"),      # one above 6
                   torch.full((1, 32), 3.4028234663852886e38, device="cuda"), torch.zeros((1, 32), device="cuda")])
    m = rt.MicroWeights(w.shape[0], 32, transposed=False, tile=1)
    ctx.micro_weights(w, m)
    # dense() is binary32: the code of the largest number of it stands for 4 x 2^126 = 2^128, which is above them all
    assert torch.equal(m.dense(), coded(w).float())
    ctx.close()


PRODUCTS = [(1, 32, 16), (1, 1500, 6000), (1, 1, 1), (2, 33, 5), (3, 1029, 515), (5, 300, 700), (8, 4096, 1024), (9, 257, 129), (24, 8192, 513), (64, 64, 64), (100, 1500, 200),
            (128, 256, 192), (129, 511, 193), (300, 2048, 1000), (700, 1500, 1030), (513, 640, 2500)]


def product_tol(x, w, depth):
    return (math.ceil(depth / 64) + 8) * 2.0 ** -22 * (x.abs() @ w.abs())


@pytest.mark.parametrize("tokens,n_in,n_out", PRODUCTS)
@pytest.mark.parametrize("ty", TYPES)
def test_micro_product(rt, tokens, n_in, n_out, ty):
    x = (normal(tokens, n_in) * torch.exp(normal(tokens, 1, seed=2))).to(ty)
    w = normal(n_out, n_in, seed=3) * 0.05
    ctx = rt.MatrixContext(rt.micro_scratch(tokens, n_out, n_in))
    for tile in (1, 32):
        m = rt.MicroWeights(n_out, n_in, transposed=False, tile=tile)
        ctx.micro_weights(w, m)
        out = torch.full((tokens, n_out), 7.0, dtype=ty, device="cuda")
        ctx.micro_product(x, m, out)
        ctx.poll_status()
        xq, wq = coded(x), coded(w, tile)
        want = xq @ wq.t()
        close(out, want, product_tol(xq, wq.t(), n_in) + rounding(ty, want))
    ctx.close()


def test_micro_product_strides(rt):
    tokens, n_in, n_out = 37, 300, 210
    base, big = normal(40, 333).bfloat16(), torch.full((40, 250), 3.0, dtype=torch.bfloat16, device="cuda")
    x, out = base[1:1 + tokens, 5:5 + n_in], big[2:2 + tokens, 7:7 + n_out]
    w = normal(n_out, n_in, seed=3)
    ctx, m = rt.MatrixContext(rt.micro_scratch(tokens, n_out, n_in)), rt.MicroWeights(n_out, n_in)
    ctx.micro_weights(w, m)
    ctx.micro_product(x, m, out)
    xq, wq = coded(x), coded(w, 32)
    want = xq @ wq.t()
    close(out, want, product_tol(xq, wq.t(), n_in) + rounding(torch.bfloat16, want))
    out.fill_(3.0)
    assert bool((big == 3.0).all())
    ctx.close()


@pytest.mark.parametrize("tokens", [1, 6, 40, 300])
def test_micro_product_of_broken_blocks(rt, tokens):
    """A NaN or an infinity in a token makes that token's results NaN, one in the weights that channel's (that tile's 32), and nothing else."""
    n_in, n_out = 200, 300
    x, w = normal(tokens, n_in), normal(n_out, n_in, seed=1)
    x[tokens // 2, 70], w[40, 100], w[290, 199] = float("nan"), float("inf"), float("nan")
    ctx, m = rt.MatrixContext(rt.micro_scratch(tokens, n_out, n_in)), rt.MicroWeights(n_out, n_in, transposed=False, tile=1)
    ctx.micro_weights(w, m)
    out = torch.zeros((tokens, n_out), device="cuda")
    ctx.micro_product(x, m, out)
    broken = torch.zeros((tokens, n_out), dtype=torch.bool, device="cuda")
    broken[tokens // 2], broken[:, 40], broken[:, 290] = True, True, True
    assert torch.equal(out.isnan(), broken)
    xq, wq = coded(x).nan_to_num(0.0), coded(w).nan_to_num(0.0)
    close(out[~broken], (xq @ wq.t())[~broken], product_tol(xq, wq.t(), n_in)[~broken])
    ctx.close()


@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 1, 1), (1, 100, 40), (31, 33, 65), (64, 128, 256), (100, 1500, 200), (257, 300, 129), (700, 513, 1030), (129, 2000, 640)])
@pytest.mark.parametrize("ty,wty", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_micro_gradients(rt, tokens, n_in, n_out, ty, wty):
    x, dy = normal(tokens, n_in).to(ty), (normal(tokens, n_out, seed=1) * 1e-3).to(ty)
    w = normal(n_out, n_in, seed=2) * 0.1
    ctx, m = rt.MatrixContext(rt.micro_scratch(tokens, n_out, n_in)), rt.MicroWeights(n_out, n_in)
    ctx.micro_weights(w, m)
    wq, rows, cols, xc = coded(w, 32), coded(dy), coded(dy, dim=0), coded(x, dim=0)
    want_x, want_w = rows @ wq, cols.t() @ xc
    tol_x = product_tol(rows, wq, n_out) + rounding(ty, want_x)
    tol_w = product_tol(cols.t(), xc, tokens) + rounding(wty, want_w)
    for both in ((True, True), (True, False), (False, True)):
        dx = torch.full((tokens, n_in), 5.0, dtype=ty, device="cuda") if both[0] else None
        dw = torch.full((n_out, n_in), 5.0, dtype=wty, device="cuda") if both[1] else None
        ctx.micro_gradients(dy, x if both[1] else None, m, dx, dw)
        ctx.poll_status()
        if dx is not None:
            close(dx, want_x, tol_x, "dx")
        if dw is not None:
            close(dw, want_w, tol_w, "dw")
    ctx.close()


def test_micro_gradients_against_differences(rt):
    """On codes that hold every operand exactly the layer is linear and its gradients are differences of its results."""
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens, n_in, n_out = 64, 96, 64

    def exact(*shape):
        v = VALUES.float().cuda()[torch.randint(0, 8, shape, generator=g, device="cuda")]
        v = v * torch.where(torch.rand(shape, generator=g, device="cuda") < 0.5, -1.0, 1.0)
        v[::16, ::16] = 6.0                     # every block's and tile's scale is 1
        v[:, ::16], v[::16, :] = 6.0, 6.0
        return v
    x, w, dy = exact(tokens, n_in), exact(n_out, n_in), exact(tokens, n_out)
    ctx, m = rt.MatrixContext(rt.micro_scratch(tokens, n_out, n_in)), rt.MicroWeights(n_out, n_in)

    def loss(x, w):
        ctx.micro_weights(w, m)
        y = torch.empty((tokens, n_out), device="cuda")
        ctx.micro_product(x, m, y)
        return float((y.double() * dy.double()).sum())
    start = loss(x, w)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ctx.micro_gradients(dy, x, m, dx, dw)
    for i, j in ((1, 1), (5, 37), (63, 95), (17, 40)):
        for v, d in ((x, dx), (w, dw)):
            moved = v.clone()
            moved[i, j] = 0.0 if float(v[i, j]) else 0.5
            other = loss(moved, w) if v is x else loss(x, moved)
            assert (other - start) == pytest.approx(float(d[i, j]) * float(moved[i, j] - v[i, j]), abs=1e-3)
    ctx.close()


# ------------------------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 64), (7, 255), (4, 256), (9, 257), (33, 1500), (20, 1029), (2, 10000), (300, 40)])
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.65, 0.999999])
def test_dropout(rt, rows, cols, ty, p):
    seed, step, worker, site = 0x123456789ABCDEF0, 0xFFFFFFFE, 65535, 32767
    base = normal(rows + 2, cols + 9).to(ty)
    mask, factor = kept(rows, cols, p, seed, step, worker, site)
    ctx = rt.MatrixContext(0)
    for x in (base[:rows, :cols].contiguous(), base[1:1 + rows, 3:3 + cols]):
        want = torch.where(mask, (x.float() * factor).to(ty), torch.zeros_like(x))
        big = torch.full((rows + 1, cols + 16), 9.0, dtype=ty, device="cuda")
        for out in (torch.full((rows, cols), 9.0, dtype=ty, device="cuda"), big[:rows, 8:8 + cols], big[1:, 5:5 + cols]):
            ctx.dropout(x, out, rt.Mask(p, seed, step, worker=worker, site=site))
            assert torch.equal(out, want)
        big[1:, 5:5 + cols] = 9.0
        big[:rows, 8:8 + cols] = 9.0
        assert bool((big == 9.0).all())
        same = x.clone()
        ctx.dropout(same, same, rt.Mask(p, seed, step, worker=worker, site=site))
        assert torch.equal(same, want)
    ctx.close()


def test_dropout_drops_whatever_it_was(rt):
    x = torch.full((4, 300), float("nan"), device="cuda")
    x[1], x[2] = float("inf"), -float("inf")
    mask, _ = kept(4, 300, 0.5, 7)
    out = torch.empty_like(x)
    ctx = rt.MatrixContext(0)
    ctx.dropout(x, out, rt.Mask(0.5, 7))
    assert torch.equal(out == 0, ~mask) and bool((out[mask] != out[mask]).sum() + out[mask].isinf().sum() == mask.sum())
    ctx.close()


# ------------------------------------------------------------------------------------------------- layer normalisation
def norm64(x, residual, gamma, beta, eps, mask):
    t = x.double()
    if mask is not None:
        t = torch.where(mask[0], t * mask[1], torch.zeros_like(t))
    if residual is not None:
        t = residual.double() + t
    mean = t.mean(1)
    rstd = (t.var(1, correction=0) + eps).rsqrt()
    h = (t - mean[:, None]) * rstd[:, None]
    y = h
    if gamma is not None:
        y = y * gamma.double()
    if beta is not None:
        y = y + beta.double()
    return t, mean, rstd, h, y


NORMS = [(1, 1), (1, 8), (3, 7), (2, 33), (5, 64), (17, 255), (8, 256), (9, 257), (20, 1500), (7, 1029), (33, 1024), (3, 2048), (4, 4097), (2, 10000), (3, 16384), (2, 20001),
         (700, 200), (1500, 96)]


@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (True, 0.3), (False, 0.5)])
def test_layer_norm(rt, rows, cols, ty, residual, p):
    eps = 1e-5
    x, res = normal(rows, cols).to(ty), (normal(rows, cols, seed=1) * 2 + normal(rows, 1, seed=2)).to(ty)
    res = res if residual else None
    gamma, beta = 1 + 0.3 * normal(cols, seed=3), normal(cols, seed=4)
    mask = kept(rows, cols, p, 11, 3, 2, 1) if p else None
    ctx = rt.MatrixContext(0)
    for g, b in ((gamma, beta), (None, None)):
        y, total = torch.full((rows, cols), 7.0, dtype=ty, device="cuda"), torch.full((rows, cols), 7.0, dtype=ty, device="cuda")
        mean, rstd = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
        ctx.layer_norm(x, g, b, y, residual=res, total=total, mean=mean, rstd=rstd, eps=eps, mask=rt.Mask(p, 11, 3, worker=2, site=1) if p else None)
        t, m, r, h, want = norm64(x, res, g, b, eps, mask)
        adds = 64 + cols / 4096
        most = t.abs().amax(1)
        d = adds * U * most * r
        close(mean, m, adds * U * most, "mean")
        close(rstd, r, r * (2 * d + adds * U), "rstd")
        close(total, t, 2 * U * (t.abs() + (res.double().abs() if residual else 0)) + rounding(ty, t), "total")
        scale = 1.0 if g is None else g.double().abs()
        tol = scale * (d[:, None] * (1 + 2 * h.abs()) + 64 * U * h.abs()) + 4 * U * want.abs() + 4 * U * (h * scale).abs()
        close(y, want, tol + rounding(ty, want), "y")
    ctx.close()


@pytest.mark.parametrize("ty", TYPES)
def test_layer_norm_strides_and_in_place(rt, ty):
    rows, cols = 13, 300
    base, rbase, obase = normal(15, 333).to(ty), normal(15, 320, seed=1).to(ty), torch.full((15, 350), 4.0, dtype=ty, device="cuda")
    x, res, out = base[1:14, 5:305], rbase[:13, 8:308], obase[1:14, 9:309]
    gamma, beta = normal(303, seed=2)[3:], normal(300, seed=3)
    ctx = rt.MatrixContext(0)
    mask, spec = kept(rows, cols, 0.25, 5), rt.Mask(0.25, 5)
    want = norm64(x, res, gamma, beta, 1e-5, mask)

    def check(y, total=None):
        close(y, want[4], 2e-4 + rounding(ty, want[4]))      # 64 u M rstd (1 + 2 |h|) |gamma| < 64 u 12 (1 + 10) 5 with these rows
        if total is not None:
            close(total, want[0], 1e-6 + rounding(ty, want[0]))
    ctx.layer_norm(x, gamma, beta, out, residual=res, mask=spec)
    check(out)
    out.fill_(4.0)
    assert bool((obase == 4.0).all())
    a, b = x.clone(), res.clone()
    ctx.layer_norm(a, gamma, beta, a, residual=b, total=b, mask=spec)      # y over x, t over the residual
    check(a, b)
    a, b = x.clone(), res.clone()
    ctx.layer_norm(a, gamma, beta, b, residual=b, total=a, mask=spec)
    check(b, a)
    ctx.close()


def test_layer_norm_of_equal_rows_and_broken_ones(rt):
    x = normal(6, 500)
    x[1], x[2], x[3, 7], x[4, 499] = 3.0, 0.0, float("nan"), float("inf")
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    beta = normal(500, seed=1)
    ctx = rt.MatrixContext(0)
    ctx.layer_norm(x, None, beta, y, mean=mean, rstd=rstd)
    # equal values: the mean is within 64 u of them, times rstd = 1 / sqrt(1e-5)
    assert bool(((y[1] - beta).abs() <= 64 * U * 3 * 317 + 4 * U * beta.abs()).all()) and torch.equal(y[2], beta)
    assert float(rstd[2]) == pytest.approx(1e5 ** 0.5, rel=1e-6)
    assert bool(y[3].isnan().all()) and bool(y[4].isnan().all())
    for i in (0, 5):
        want = norm64(x[i:i + 1], None, None, beta, 1e-5, None)[4][0]
        close(y[i], want, 64 * U * 4 * 5 + 64 * U * want.abs())
    ctx.close()


def back64(dy, total, mean, rstd, gamma, dtotal, mask):
    dy, h = dy.double(), (total.double() - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy if gamma is None else dy * gamma.double()
    d = rstd.double()[:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    if dtotal is not None:
        d = d + dtotal.double()
    dx = d if mask is None else torch.where(mask[0], d * mask[1], torch.zeros_like(d))
    return d, dx, dy * h, dy


@pytest.mark.parametrize("rows,cols", NORMS + [(5000, 72), (3000, 515), (2600, 2048)])
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("dtotal,p", [(False, 0.0), (True, 0.0), (True, 0.3)])
def test_layer_norm_gradients(rt, rows, cols, ty, dtotal, p):
    total = (normal(rows, cols) * 2 + normal(rows, 1, seed=2)).to(ty)
    dy, dt = normal(rows, cols, seed=1).to(ty), normal(rows, cols, seed=5).to(ty) if dtotal else None
    gamma = 1 + 0.3 * normal(cols, seed=3)
    mean = total.double().mean(1).float()
    rstd = (total.double().var(1, correction=0) + 1e-5).rsqrt().float()
    mask = kept(rows, cols, p, 21, 4, 1, 9) if p else None
    spec = rt.Mask(p, 21, 4, worker=1, site=9) if p else None
    ctx = rt.MatrixContext(rt.layer_norm_scratch(rows, cols))
    for g in (gamma, None):
        dr = torch.full((rows, cols), 7.0, dtype=ty, device="cuda")
        dx = torch.full((rows, cols), 7.0, dtype=ty, device="cuda") if p else None
        dgamma, dbeta = torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
        ctx.layer_norm_gradients(dy, total, mean, rstd, g, dr, dgamma=dgamma, dbeta=dbeta, dtotal=dt, dx=dx, mask=spec)
        d, wx, wg, wb = back64(dy, total, mean, rstd, g, dt, mask)
        h = (total.double() - mean.double()[:, None]) * rstd.double()[:, None]
        gg = (dy.double() if g is None else dy.double() * g.double()).abs()
        eh = 4 * U * (total.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None] + 4 * U * h.abs()
        adds = (64 + cols / 4096) * U
        along = (gg * h.abs()).mean(1, keepdim=True)
        tol = rstd.double()[:, None] * (4 * U * gg + adds * gg.mean(1, keepdim=True) + h.abs() * (adds * along + (gg * eh).mean(1, keepdim=True)) + eh * along)
        tol = tol + 4 * U * d.abs() + 4 * U * ((dt.double().abs() if dtotal else 0) + rstd.double()[:, None] * (gg + along * h.abs()))
        close(dr, d, tol + rounding(ty, d), "dresidual")
        if p:
            close(dx, wx, torch.where(mask[0], tol * mask[1] + rounding(ty, wx) + 2 * U * wx.abs(), torch.zeros_like(tol)), "dx")
        adds = (64 + rows / 4096) * U
        close(dgamma, wg.sum(0), adds * wg.abs().sum(0) + (dy.double().abs() * eh).sum(0) + U * wg.sum(0).abs(), "dgamma")
        close(dbeta, wb.sum(0), adds * wb.abs().sum(0), "dbeta")
        again = torch.empty_like(dgamma)
        ctx.layer_norm_gradients(dy, total, mean, rstd, g, dgamma=again)
        assert torch.equal(again, dgamma)
    ctx.close()


def test_layer_norm_gradients_in_place_and_with_strides(rt):
    rows, cols = 41, 300
    ctx = rt.MatrixContext(rt.layer_norm_scratch(rows, cols))
    for ty in TYPES:
        b = [normal(44, 333, seed=i).to(ty) for i in range(3)]
        dy, total, dt = b[0][1:42, 5:305], b[1][:41, 8:308], b[2][2:43, 1:301]
        mean, rstd = total.double().mean(1).float(), (total.double().var(1, correction=0) + 1e-5).rsqrt().float()
        mask, spec = kept(rows, cols, 0.25, 5), rt.Mask(0.25, 5)
        d, wx, wg, wb = back64(dy, total, mean, rstd, None, dt, mask)
        tol = 64 * U * 60                      # rstd (|g| + mean |g| + |h| mean |g h|) is below 60 with these rows
        for first, second in ((0, 2), (2, 0)):      # dresidual over dy and dx over dtotal, and the other way round
            c = [v.clone() for v in (dy, total, dt)]
            dgamma, dbeta = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
            ctx.layer_norm_gradients(c[0], c[1], mean, rstd, None, c[first], dgamma=dgamma, dbeta=dbeta, dtotal=c[2], dx=c[second], mask=spec)
            close(c[first], d, tol + rounding(ty, d))
            close(c[second], wx, 2 * tol + rounding(ty, wx))
            close(dgamma, wg.sum(0), 64 * U * wg.abs().sum(0) + 64 * U * 60)
            close(dbeta, wb.sum(0), 64 * U * wb.abs().sum(0))
    ctx.close()


def test_layer_norm_gradients_against_differences(rt):
    """The forward pass in 32 bits at a distance of 2^-7: central differences are off by their third derivatives (about 2^-14 / 6 times a
    few of them, each below 8 here) and by roundings of the sum over 2^-7, both below 2e-3."""
    rows, cols, step = 3, 40, 2.0 ** -7
    x, res, gamma, beta, dy, dt = (normal(rows, cols, seed=i) for i in range(2)), None, 1 + 0.2 * normal(cols, seed=3), normal(cols, seed=4), normal(rows, cols, seed=5), normal(rows, cols, seed=6)
    x, res = x
    ctx, spec = rt.MatrixContext(rt.layer_norm_scratch(rows, cols)), rt.Mask(0.3, 77, 1)
    y, total, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def loss(x, res, gamma, beta):
        ctx.layer_norm(x, gamma, beta, y, residual=res, total=total, mean=mean, rstd=rstd, mask=spec)
        return float((y.double() * dy.double()).sum() + (total.double() * dt.double()).sum())
    loss(x, res, gamma, beta)
    dr, dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    ctx.layer_norm_gradients(dy, total, mean, rstd, gamma, dr, dgamma=dgamma, dbeta=dbeta, dtotal=dt, dx=dx, mask=spec)
    args = [x, res, gamma, beta]
    for which, grad in enumerate((dx, dr, dgamma, dbeta)):
        for at in (0, 17, cols - 1):
            i = (1, at) if which < 2 else (at,)
            ends = []
            for sign in (1, -1):
                moved = [v.clone() for v in args]
                moved[which][i] += sign * step
                ends.append(loss(*moved))
            assert (ends[0] - ends[1]) / (2 * step) == pytest.approx(float(grad[i]), abs=2e-3)
    ctx.close()


# ------------------------------------------------------------------------------------------------- together
def test_no_rows(rt):
    ctx = rt.MatrixContext(0)
    x, y = torch.empty((0, 40), device="cuda"), torch.empty((0, 24), device="cuda")
    m = rt.MicroWeights(24, 40)
    ctx.micro_product(x, m, y)
    ctx.dropout(x, x, rt.Mask(0.5, 1))
    ctx.layer_norm(x, None, None, x)
    dw = torch.full((24, 40), 5.0, device="cuda")
    ctx.micro_gradients(y, x, m, x, dw)
    dgamma, dbeta = torch.full((40,), 5.0, device="cuda"), torch.full((40,), 5.0, device="cuda")
    e = torch.empty(0, device="cuda")
    ctx.layer_norm_gradients(x, x, e, e, None, x, dgamma=dgamma, dbeta=dbeta)
    assert bool((dw == 0).all()) and bool((dgamma == 0).all()) and bool((dbeta == 0).all())
    ctx.close()


def test_refusals(rt):
    ctx = rt.MatrixContext(1024)
    x, y, w = normal(70, 40), normal(70, 24), normal(24, 40)
    m = rt.MicroWeights(24, 40)
    ctx.micro_weights(w, m)
    e = rt.RTopKError
    for call, error in [(lambda: ctx.micro_product(x, m, y), e),                                     # too little scratch
                        (lambda: ctx.micro_gradients(y, x, m, x), e),
                        (lambda: ctx.micro_gradients(y, x, m), e),                                   # nothing asked for
                        (lambda: ctx.micro_gradients(y, None, m, dw=w), ValueError),
                        (lambda: ctx.micro_gradients(y, x, rt.MicroWeights(24, 40, transposed=False), x), ValueError),
                        (lambda: ctx.micro_product(x.half(), m, y.half()), TypeError),
                        (lambda: ctx.micro_product(x, m, y.bfloat16()), TypeError),
                        (lambda: ctx.micro_product(x.cpu(), m, y), ValueError),
                        (lambda: ctx.micro_product(x[:, :39], m, y), ValueError),
                        (lambda: ctx.dropout(x, y, rt.Mask(0.5, 1)), ValueError),
                        (lambda: ctx.dropout(x, x, None), e),
                        (lambda: ctx.dropout(x, x.bfloat16(), rt.Mask(0.5, 1)), TypeError),
                        (lambda: ctx.dropout(x, x, rt.Mask(0.5, 1, torch.zeros(1, dtype=torch.int32))), ValueError),      # a step of the CPU's
                        (lambda: rt.Mask(1.0, 1), ValueError), (lambda: rt.Mask(float("nan"), 1), ValueError), (lambda: rt.Mask(0.5, 1, worker=65536), ValueError),
                        (lambda: rt.Mask(0.5, 1, torch.zeros(1, device="cuda")), ValueError),
                        (lambda: ctx.layer_norm(x, w[0, :39], None, x), ValueError),
                        (lambda: ctx.layer_norm(x, w[0].bfloat16(), None, x), TypeError),
                        (lambda: ctx.layer_norm(x, None, None, x, eps=-1.0), e), (lambda: ctx.layer_norm(x, None, None, x, eps=float("nan")), e),
                        (lambda: ctx.layer_norm(x, None, None, x, residual=y), ValueError),
                        (lambda: ctx.layer_norm(x, None, None, x.t().contiguous().t()), ValueError),
                        (lambda: ctx.layer_norm_gradients(x, x, None, None, None, x), e),
                        (lambda: ctx.layer_norm_gradients(x, x, x[:, 0].contiguous(), x[:, 0].contiguous(), None, x, dx=x), ValueError),
                        (lambda: ctx.layer_norm_gradients(x, x, x[:, 0].contiguous(), x[:, 0].contiguous(), None), e)]:
        with pytest.raises(error):
            call()
    big = rt.MatrixContext(0)
    s = torch.zeros(70, device="cuda")
    with pytest.raises(e):                                                                            # no scratch for the sums over rows
        big.layer_norm_gradients(x, x, s, s, None, x.clone(), dgamma=torch.zeros(40, device="cuda"))
    big.layer_norm_gradients(x, x, s, s, None, x.clone())
    torch.cuda.synchronize()
    ctx.close()
    big.close()


def block(rt, ctx, p, io):
    """A residual block of a worker, forwards and backwards, on buffers that `io` holds."""
    ctx.layer_norm(io["x"], io["g1"], io["b1"], io["n1"], mean=io["m1"], rstd=io["r1"])
    ctx.micro_product(io["n1"], io["w1"], io["h"])
    torch.clamp(io["h"], min=0, out=io["a"])
    ctx.micro_product(io["a"], io["w2"], io["o"])
    ctx.layer_norm(io["o"], io["g2"], io["b2"], io["y"], residual=io["x"], total=io["t"], mean=io["m2"], rstd=io["r2"], mask=p)
    ctx.layer_norm_gradients(io["dy"], io["t"], io["m2"], io["r2"], io["g2"], io["dr"], dgamma=io["dg2"], dbeta=io["db2"], dx=io["do"], mask=p)
    ctx.micro_gradients(io["do"], io["a"], io["w2"], io["da"], io["dw2"])
    torch.mul(io["da"], io["h"] > 0, out=io["dh"])
    ctx.micro_gradients(io["dh"], io["n1"], io["w1"], io["dn"], io["dw1"])
    ctx.layer_norm_gradients(io["dn"], io["x"], io["m1"], io["r1"], io["g1"], io["dx"], dgamma=io["dg1"], dbeta=io["db1"], dtotal=io["dr"])


def block_buffers(rt, ctx, tokens, d, hidden, ty, seed):
    def empty(*shape, dtype=ty):
        return torch.zeros(shape, dtype=dtype, device="cuda")
    io = {"x": normal(tokens, d, seed=seed).to(ty), "dy": normal(tokens, d, seed=seed + 1).to(ty) * 1e-2}
    for k in ("n1", "o", "y", "t", "dr", "do", "dn", "dx"):
        io[k] = empty(tokens, d)
    for k in ("h", "a", "da", "dh"):
        io[k] = empty(tokens, hidden)
    for k in ("m1", "r1", "m2", "r2"):
        io[k] = empty(tokens, dtype=torch.float32)
    for k in ("dg1", "db1", "dg2", "db2"):
        io[k] = empty(d, dtype=torch.float32)
    for i, k in enumerate(("g1", "g2")):
        io[k] = 1 + 0.1 * normal(d, seed=seed + 2 + i)
    for i, k in enumerate(("b1", "b2")):
        io[k] = 0.1 * normal(d, seed=seed + 4 + i)
    io["w1"], io["w2"] = rt.MicroWeights(hidden, d), rt.MicroWeights(d, hidden)
    for i, w in enumerate((io["w1"], io["w2"])):
        ctx.micro_weights(normal(w.n_out, w.n_in, seed=seed + 6 + i) / w.n_in ** 0.5, w)
    io["dw1"], io["dw2"] = empty(hidden, d, dtype=torch.float32), empty(d, hidden, dtype=torch.float32)
    return io


RESULTS = ("y", "t", "dx", "dw1", "dw2", "dg1", "db1", "dg2", "db2")


@pytest.mark.parametrize("tokens,d,hidden,ty", [(70, 96, 200, torch.float32), (300, 515, 1029, torch.bfloat16), (1, 64, 64, torch.float32)])
def test_a_block_forwards_and_backwards_on_streams_and_in_graphs(rt, tokens, d, hidden, ty):
    """Each step equals its definition on what the step before gave (the tests above); here: the same bits every time, on another stream and
    from a graph whose replays take the round number from the device."""
    need = max(rt.micro_scratch(tokens, hidden, d), rt.layer_norm_scratch(tokens, d))
    ctx = rt.MatrixContext(need)
    io = block_buffers(rt, ctx, tokens, d, hidden, ty, 40)
    by_step = {}
    for step in (3, 4, 9):
        block(rt, ctx, rt.Mask(0.2, 99, step, worker=1), io)
        by_step[step] = {k: io[k].clone() for k in RESULTS}
    assert tokens == 1 or not torch.equal(by_step[3]["t"], by_step[4]["t"])
    mask, factor = kept(tokens, d, 0.2, 99, 9, 1)
    want = norm64(io["o"], io["x"], io["g2"], io["b2"], 1e-5, (mask, factor))
    close(io["y"], want[4], 2e-4 + rounding(ty, want[4]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(rt, ctx, rt.Mask(0.2, 99, 4, worker=1), io)
    side.synchronize()
    for k in RESULTS:
        assert torch.equal(io[k], by_step[4][k]), k
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block(rt, ctx, rt.Mask(0.2, 99, step, worker=1), io)
    for s in (9, 3, 4):
        step.fill_(s)
        graph.replay()
        torch.cuda.synchronize()
        for k in RESULTS:
            assert torch.equal(io[k], by_step[s][k]), (s, k)
    ctx.poll_status()
    ctx.close()
