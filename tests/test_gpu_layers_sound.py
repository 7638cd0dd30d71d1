"""A worker's layers in calls that once went wrong.  Tolerances as derived in test_gpu_layers.py (u = 2^-24) unless a test says otherwise."""
import numpy as np
import pytest
import torch

from test_gpu_layers import TYPES, U, back64, close, normal, rounding, rt  # noqa: F401

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
