"""A worker's layers in calls that once went wrong or that no test made.  Tolerances as derived in test_gpu_layers.py (u = 2^-24) unless a test says otherwise."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import test_gpu_layers as base
from test_gpu_layers import TYPES, U, back64, close, norm64, normal, rounding, rt  # noqa: F401

pytestmark = pytest.mark.gpu


def kept_from(col0, cols, row, p, seed, step=0):
    """As `kept`, of one row's columns from col0 (a multiple of eight) on."""
    u, g = np.uint64, -(-cols // 8)
    c = [np.arange(col0 // 8, col0 // 8 + g, dtype=u), np.full(g, row, dtype=u), np.full(g, 1 << 31, dtype=u), np.full(g, step, dtype=u)]
    for i in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        k0, k1 = u((seed + i * 0x9E3779B9) % 2 ** 32), u(((seed >> 32) + i * 0xBB67AE85) % 2 ** 32)
        c = [(b >> u(32)) ^ c[1] ^ k0, b & u(0xFFFFFFFF), (a >> u(32)) ^ c[3] ^ k1, a & u(0xFFFFFFFF)]
    numbers = np.stack(c, 1).astype(np.uint32).view(np.uint16).reshape(-1)[:cols]
    return torch.from_numpy(numbers >= round(65536 * p)).cuda()


@pytest.mark.parametrize("ty,rows,cols", [(torch.bfloat16, 1, 1 << 26), (torch.bfloat16, 5, (1 << 26) + 8), (torch.float32, 1, 100000000), (torch.bfloat16, 9, (1 << 27) + 24),
                                          (torch.bfloat16, 2, (1 << 26) + 3)])
def test_dropout_of_very_wide_rows(rt, ty, rows, cols):  # noqa: F811
    p, seed = 0.25, 0xABCDEF0123456789
    factor = float(np.float32(65536 / 49152))
    x = torch.empty((rows, cols), dtype=ty, device="cuda")
    x.view(-1)[:1 << 20] = 1 + torch.rand(1 << 20, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(ty)
    flat = x.view(-1)
    for at in range(1 << 20, rows * cols, 1 << 20):
        flat[at:at + (1 << 20)] = flat[:min(1 << 20, rows * cols - at)]
    ctx, spec = rt.MatrixContext(0), rt.Mask(p, seed, 6)
    out = torch.full_like(x, 7.0)
    ctx.dropout(x, out, spec)
    places = [(0, 1000), (cols // 16 * 8, 1000), ((cols - 700) // 8 * 8, cols - (cols - 700) // 8 * 8)]
    for row in {0, rows // 2, rows - 1}:
        for at, n in places:
            v = x[row, at:at + n]
            assert torch.equal(out[row, at:at + n], torch.where(kept_from(at, n, row, p, seed, 6), (v.float() * factor).to(ty), torch.zeros_like(v))), (row, at)
        # elsewhere: dropped or scaled, and dropped as often as p says (8 standard deviations)
        dropped = 0
        for at in range(0, cols, 1 << 24):
            o, v = out[row, at:at + (1 << 24)], x[row, at:at + (1 << 24)]
            zero = o == 0
            assert bool((zero | (o == (v.float() * factor).to(ty))).all())
            dropped += int(zero.sum())
        assert abs(dropped - p * cols) < 8 * (p * (1 - p) * cols) ** 0.5
    ctx.dropout(x, x, spec)
    assert torch.equal(x, out)
    ctx.close()


# ------------------------------------------------------------------------------------------------- large means
@pytest.mark.parametrize("rows,cols", [(700, 200), (64, 256), (700, 1500), (300, 1504), (170, 4096), (170, 4099), (160, 10000), (40, 16384), (5, 20001)])
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("far", [10.0, 1000.0])
def test_layer_norm_gradients_of_rows_with_large_means(rt, rows, cols, ty, far):  # noqa: F811
    """With mean and rstd given, h = (total - mean) rstd has two roundings: it is within 2 u of itself, whatever the mean is."""
    total = (normal(rows, cols) + far * (1 + normal(rows, 1, seed=2).abs())).to(ty)
    dy, gamma = normal(rows, cols, seed=1).to(ty), 1 + 0.3 * normal(cols, seed=3)
    mean = total.double().mean(1).float()
    rstd = (total.double().var(1, correction=0) + 1e-5).rsqrt().float()
    ctx = rt.MatrixContext(rt.layer_norm_scratch(rows, cols))
    dr, dgamma, dbeta = torch.full((rows, cols), 7.0, dtype=ty, device="cuda"), torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    ctx.layer_norm_gradients(dy, total, mean, rstd, gamma, dr, dgamma=dgamma, dbeta=dbeta)
    d, _, wg, wb = back64(dy, total, mean, rstd, gamma, None, None)
    r = rstd.double()[:, None]
    h = (total.double() - mean.double()[:, None]) * r
    gg, eh = (dy.double() * gamma.double()).abs(), 2.01 * U * h.abs()
    adds = (64 + cols / 4096) * U
    along = (gg * h.abs()).mean(1, keepdim=True)
    tol = r * (4 * U * gg + adds * gg.mean(1, keepdim=True) + h.abs() * (adds * along + (gg * eh).mean(1, keepdim=True)) + eh * along)
    tol = tol + 4 * U * d.abs() + 4 * U * r * (gg + along * h.abs())
    close(dr, d, tol + rounding(ty, d), "dresidual")
    adds = (64 + rows / 4096) * U
    close(dgamma, wg.sum(0), adds * wg.abs().sum(0) + (dy.double().abs() * eh).sum(0) + U * wg.sum(0).abs(), "dgamma")
    close(dbeta, wb.sum(0), adds * wb.abs().sum(0), "dbeta")
    ctx.close()


# ------------------------------------------------------------------------------------------------- the ends of the range
@pytest.mark.parametrize("cols", [1, 200, 1500, 1504, 10000, 20001])
@pytest.mark.parametrize("ty", TYPES)
def test_layer_norm_at_the_ends_of_the_range(rt, cols, ty):  # noqa: F811
    """1 / sqrt is 0 of infinity and infinity of 0: finite rows whose squares leave binary32 come out as beta, and without an eps a row whose
    variance is 0 has an infinite rstd, and no results."""
    ctx = rt.MatrixContext(rt.layer_norm_scratch(4, cols))
    x = normal(4, cols).to(ty)
    x[1] = torch.where(torch.arange(cols, device="cuda") % 2 == 0, 3e30, -3e30).to(ty)
    x[2] = 3.0
    gamma, beta = 1 + 0.3 * normal(cols, seed=3), normal(cols, seed=4)
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    for eps in (1e-5, 0.0):
        ctx.layer_norm(x, gamma, beta, y, mean=mean, rstd=rstd, eps=eps)
        if cols > 1:
            assert float(rstd[1]) == 0.0 and bool(mean[1].isfinite())
            assert torch.equal(y[1], beta.to(ty))
        if eps == 0.0:      # equal values: mean and differences are within adds u of them, so the variance is at most the square of that
            adds = 64 + cols / 4096
            assert float(rstd[2]) >= (1 - adds * U) / (adds * U * 3)
        if cols > 1:
            for i in (0, 3):
                t, m, r, h, want = norm64(x[i:i + 1], None, gamma, beta, eps, None)
                adds = 64 + cols / 4096
                d = adds * U * t.abs().amax(1) * r
                close(rstd[i:i + 1], r, r * (2 * d + adds * U))
                tol = gamma.double().abs() * (d[:, None] * (1 + 2 * h.abs()) + 64 * U * h.abs()) + 4 * U * want.abs() + 4 * U * (h * gamma.double()).abs()
                close(y[i:i + 1], want, tol + rounding(ty, want))
    x[2] = 0.0
    ctx.layer_norm(x, gamma, beta, y, rstd=rstd, eps=0.0)
    assert float(rstd[2]) == float("inf") and bool(y[2].isnan().all())
    # the gradients of the rows with rstd = 0: what reaches t on its other way, and nothing for gamma
    dy, dt = normal(4, cols, seed=5).to(ty), normal(4, cols, seed=6).to(ty)
    m1, zero = x[1].double().mean().float().expand(4).contiguous(), torch.zeros(4, device="cuda")
    dr, dgamma = torch.empty_like(x), torch.empty(cols, device="cuda")
    rows = x[1:2].expand(4, cols).contiguous()
    ctx.layer_norm_gradients(dy, rows, m1, zero, gamma, dr, dgamma=dgamma, dtotal=dt)
    assert torch.equal(dr, dt) and not bool(dgamma.any())
    ctx.close()


@pytest.mark.parametrize("cols", [3, 200, 256, 1500, 1504, 10000, 20001])
@pytest.mark.parametrize("ty", TYPES)
def test_layer_norm_gradients_of_huge_equal_rows(rt, cols, ty):  # noqa: F811
    """h is 0 in every column; a column that is not there, with a total of 0, would have -mean rstd, beyond binary32."""
    rows, rstd = 300, torch.full((300,), 1e6, device="cuda")      # eps = 1e-12
    total = torch.full((rows, cols), 1e33, device="cuda").to(ty)
    mean = total[:, 0].float().contiguous()
    dy = normal(rows, cols, seed=1).to(ty)
    ctx = rt.MatrixContext(rt.layer_norm_scratch(rows, cols))
    dr, dgamma, dbeta = torch.empty_like(dy), torch.full((cols,), 7.0, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    ctx.layer_norm_gradients(dy, total, mean, rstd, None, dr, dgamma=dgamma, dbeta=dbeta)
    g = dy.double()
    want = 1e6 * (g - g.mean(1, keepdim=True))
    close(dr, want, 1e6 * ((64 + cols / 4096) * U * g.abs().mean(1, keepdim=True) + 4 * U * g.abs()) + 4 * U * want.abs() + rounding(ty, want))
    assert not bool(dgamma.any())
    close(dbeta, g.sum(0), 65 * U * g.abs().sum(0))
    ctx.close()


# ------------------------------------------------------------------------------------------------- long rows
@pytest.mark.parametrize("cols", [(1 << 24) + 8, (1 << 24) + 1])
def test_long_rows_of_equal_values(rt, cols):  # noqa: F811
    """Sums of equal terms lose the most: each addition's rounding has the same sign."""
    rows, v = 2, 0.5141598582267761
    x = torch.full((rows, cols), v, device="cuda")
    x[1, 1::2] = -v
    adds = (64 + cols / 4096) * U
    ctx = rt.MatrixContext(rt.layer_norm_scratch(rows, cols))
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ctx.layer_norm(x, None, None, y, mean=mean, rstd=rstd)
    t, m, r, h, want = norm64(x, None, None, None, 1e-5, None)
    d = adds * v * r
    close(mean, m, torch.full_like(m, adds * v), "mean")
    close(rstd, r, r * (2 * d + adds), "rstd")
    close(y, want, d[:, None] * (1 + 2 * h.abs()) + 64 * U * h.abs() + 8 * U * want.abs(), "y")
    # gradients: equal terms in the sums of g, then of g h
    mean, rstd = m.float(), r.float()
    dr = torch.empty_like(x)
    for dy in (torch.full_like(x, v), x):
        ctx.layer_norm_gradients(dy, x, mean, rstd, None, dr)
        d, _, _, _ = back64(dy, x, mean, rstd, None, None, None)
        r1, h = rstd.double()[:, None], (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        gg = dy.double().abs()
        eh, along = 2.01 * U * h.abs(), (gg * h.abs()).mean(1, keepdim=True)
        tol = r1 * (4 * U * gg + adds * gg.mean(1, keepdim=True) + h.abs() * (adds * along + (gg * eh).mean(1, keepdim=True)) + eh * along)
        close(dr, d, tol + 4 * U * d.abs() + 4 * U * r1 * (gg + along * h.abs()), "dresidual")
    ctx.close()


# ------------------------------------------------------------------------------------------------- wide rows, several to a block
@pytest.mark.parametrize("cols", [10000, 16384])
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (True, 0.3)])
def test_blocks_that_take_several_wide_rows(rt, cols, ty, residual, p):  # noqa: F811
    rows = 700
    base.test_layer_norm(rt, rows, cols, ty, residual, p)
    base.test_layer_norm_gradients(rt, rows, cols, ty, residual, p)
    # the same bits in place
    ctx, spec = rt.MatrixContext(0), rt.Mask(p, 11, 3) if p else None
    x, res, gamma = normal(rows, cols).to(ty), normal(rows, cols, seed=1).to(ty) if residual else None, 1 + 0.3 * normal(cols, seed=3)
    y, total, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ctx.layer_norm(x, gamma, None, y, residual=res, total=total, mean=mean, rstd=rstd, mask=spec)
    a, b = x.clone(), res.clone() if residual else torch.empty_like(x)
    ctx.layer_norm(a, gamma, None, a, residual=b if residual else None, total=b, mask=spec)
    assert torch.equal(a, y) and torch.equal(b, total)
    dy, dt = normal(rows, cols, seed=5).to(ty), normal(rows, cols, seed=6).to(ty) if residual else None
    dr, dx = torch.empty_like(x), torch.empty_like(x) if p else None
    ctx.layer_norm_gradients(dy, total, mean, rstd, gamma, dr, dtotal=dt, dx=dx, mask=spec)
    a, b = dy.clone(), dt.clone() if residual else None
    ctx.layer_norm_gradients(a, total, mean, rstd, gamma, a, dtotal=b, dx=b if p else None, mask=spec)
    assert torch.equal(a, dr) and (not p or torch.equal(b, dx))
    ctx.close()


def test_two_contexts_at_once(rt):  # noqa: F811
    """Blocks of two workers on streams of their own, eager and replayed: the same bits as one after another."""
    workers, spec = [], rt.Mask(0.2, 99, 4, worker=1)
    for tokens, d, hidden, ty, seed in ((300, 515, 1029, torch.bfloat16, 40), (700, 1024, 2048, torch.float32, 80)):
        ctx = rt.MatrixContext(max(rt.micro_scratch(tokens, hidden, d), rt.layer_norm_scratch(tokens, d)))
        io = base.block_buffers(rt, ctx, tokens, d, hidden, ty, seed)
        base.block(rt, ctx, spec, io)
        torch.cuda.synchronize()
        want = {k: io[k].clone() for k in base.RESULTS}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            base.block(rt, ctx, spec, io)
        workers.append((ctx, io, want, torch.cuda.Stream(), graph))
    for replayed in (False, True):
        for _, io, _, _, _ in workers:
            for k in base.RESULTS:
                io[k].fill_(5.0)
        torch.cuda.synchronize()
        for _ in range(30):
            for ctx, io, _, stream, graph in workers:
                with torch.cuda.stream(stream):
                    if replayed:
                        graph.replay()
                    else:
                        base.block(rt, ctx, spec, io)
        torch.cuda.synchronize()
        for ctx, io, want, _, _ in workers:
            ctx.poll_status()
            for k in base.RESULTS:
                assert torch.equal(io[k], want[k]), (replayed, k)
    while workers:
        workers.pop()[0].close()


FIRST = """
import torch
import paper_2005_10761_b200 as rt
tokens, d, hidden = 70, 96, 200
def buffers():
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((tokens, d), generator=g, device="cuda").to(ty) for _ in range(2))
    io = dict(x=x, dy=dy, w=torch.randn((d, d), generator=g, device="cuda"), m=rt.MicroWeights(d, d))
    for k in "o1", "h", "y", "t", "dr", "dh", "dx":
        io[k] = torch.zeros_like(x)
    io["o1"] = io["o1"][:1]
    for k, n in (("mean", tokens), ("rstd", tokens), ("dgamma", d), ("dbeta", d)):
        io[k] = torch.zeros(n, device="cuda")
    io["dw"] = torch.zeros((d, d), device="cuda")
    return io
def calls(ctx, io):
    spec = rt.Mask(0.2, 9, 1)
    ctx.micro_weights(io["w"], io["m"])
    ctx.micro_product(io["x"][:1], io["m"], io["o1"])
    ctx.micro_product(io["x"], io["m"], io["h"])
    ctx.dropout(io["h"], io["h"], spec)
    ctx.layer_norm(io["h"], None, None, io["y"], residual=io["x"], total=io["t"], mean=io["mean"], rstd=io["rstd"], mask=spec)
    ctx.layer_norm_gradients(io["dy"], io["t"], io["mean"], io["rstd"], None, io["dr"], dgamma=io["dgamma"], dbeta=io["dbeta"], dtotal=io["x"], dx=io["dh"], mask=spec)
    ctx.micro_gradients(io["dh"], io["x"], io["m"], io["dx"], io["dw"])
for ty in torch.float32, torch.bfloat16:
    io, again = buffers(), buffers()
    ctx = rt.MatrixContext(max(rt.micro_scratch(tokens, d, d), rt.layer_norm_scratch(tokens, d)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(ctx, io)
    graph.replay()
    torch.cuda.synchronize()
    ctx.poll_status()
    calls(ctx, again)
    torch.cuda.synchronize()
    for k in io:
        if isinstance(io[k], torch.Tensor):
            assert torch.equal(io[k], again[k]) and bool(io[k].any()), k
    del graph
    ctx.close()
print("as later calls")
"""


def test_the_first_calls_of_a_process_may_be_captured(rt):  # noqa: F811
    """Kernels are loaded and given their shared memory at a context's first call of their kind, in a capture too."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    ran = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert ran.returncode == 0 and ran.stdout.strip() == "as later calls", ran.stdout + ran.stderr
