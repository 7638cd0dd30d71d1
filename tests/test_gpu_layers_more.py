"""A worker's layers at the edges: scales at both ends of the range, long and distant rows, scratch of just the size, blocks that give up."""
import ctypes
import copy
import time

import pytest
import torch

from test_gpu_layers import TYPES, U, back64, close, coded, kept, norm64, normal, product_tol, rounding, rt  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 2, 4, 7, 30, 300])
def test_micro_product_with_scales_at_both_ends(rt, tokens):  # noqa: F811
    """Tokens around 2^-110, 1 and 2^110 through weights around 2^100, 1 and 2^-100, wherever the results stay within binary32's normal numbers: a
    token's scales and a channel's are powers of two, so every result is that power times the same sum as without them."""
    n_in, n_out = 160, 200
    x, w = normal(tokens, n_in), normal(n_out, n_in, seed=1)
    powers_x = [(-110, 0, 110)[(i + tokens) % 3] for i in range(tokens)]
    powers_w = [(100, 0, -100)[i // 32 % 3] for i in range(n_out)]
    px = torch.tensor([2.0 ** p for p in powers_x], device="cuda")[:, None]
    pw = torch.tensor([2.0 ** p for p in powers_w], device="cuda")[:, None]
    ctx, m = rt.MatrixContext(rt.micro_scratch(tokens, n_out, n_in)), rt.MicroWeights(n_out, n_in)
    ctx.micro_weights(w * pw, m)
    out = torch.empty((tokens, n_out), device="cuda")
    ctx.micro_product(x * px, m, out)
    xq, wq = coded(x), coded(w, 32)
    power = px.double() * pw.double().t()
    want, tol = (xq @ wq.t()) * power, product_tol(xq, wq.t(), n_in) * power
    inside = (power > 2.0 ** -115) & (power < 2.0 ** 115)
    # past the range there is an infinity, or the NaN of blocks that are infinities of both signs: no finite number, but where the exact sum is zero
    beyond = ~inside & (power > 1) & (want != 0)
    assert bool(inside.any()) and bool((want[beyond].abs() >= 2.0 ** 128).all()) and not bool(out[beyond].isfinite().any())
    close(out[inside], want[inside], tol[inside])
    ctx.close()


def test_micro_codes_of_bfloat16_at_the_ends_of_the_range(rt):  # noqa: F811
    bits = torch.arange(0, 0x7F80, 7, device="cuda", dtype=torch.int32)
    row = (bits << 16).view(torch.float32)
    w = torch.stack([row.repeat(2)[:4096], -row.flip(0).repeat(2)[:4096]]).bfloat16()
    w = torch.cat([w, torch.full((1, 4096), 2.0 ** -133, device="cuda").bfloat16(), torch.zeros((1, 4096), device="cuda").bfloat16()])
    w[2, 31], w[2, 64 + 5], w[3, 100] = float("nan"), float("inf"), -float("inf")
    ctx, m = rt.MatrixContext(0), rt.MicroWeights(4, 4096, transposed=False, tile=1)
    ctx.micro_weights(w, m)
    want = coded(w).float()
    assert torch.equal(m.dense().isnan(), want.isnan()) and torch.equal(m.dense().nan_to_num(0.0), want.nan_to_num(0.0))
    ctx.close()


@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 70001, 130), (3, 300000, 16), (40, 200001, 24)])
def test_micro_products_over_long_rows(rt, tokens, n_in, n_out):  # noqa: F811
    x, w = normal(tokens, n_in), normal(n_out, n_in, seed=1)
    ctx, m = rt.MatrixContext(rt.micro_scratch(tokens, n_out, n_in)), rt.MicroWeights(n_out, n_in)
    ctx.micro_weights(w, m)
    out, dx, dw = torch.empty((tokens, n_out), device="cuda"), torch.empty_like(x), torch.empty_like(w)
    ctx.micro_product(x, m, out)
    xq, wq = coded(x), coded(w, 32)
    close(out, xq @ wq.t(), product_tol(xq, wq.t(), n_in))
    dy = normal(tokens, n_out, seed=2)
    ctx.micro_gradients(dy, x, m, dx, dw)
    rows, cols, xc = coded(dy), coded(dy, dim=0), coded(x, dim=0)
    close(dx, rows @ wq, product_tol(rows, wq, n_out))
    close(dw, cols.t() @ xc, product_tol(cols.t(), xc, tokens))
    ctx.poll_status()
    ctx.close()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("cols", [40000, 70001])
def test_long_rows(rt, ty, cols):  # noqa: F811
    rows = 3
    x, res, dy = normal(rows, cols).to(ty), normal(rows, cols, seed=1).to(ty), normal(rows, cols, seed=2).to(ty)
    gamma, beta = 1 + 0.2 * normal(cols, seed=3), normal(cols, seed=4)
    mask, spec = kept(rows, cols, 0.2, 9), rt.Mask(0.2, 9)
    ctx = rt.MatrixContext(rt.layer_norm_scratch(rows, cols))
    y, total, dr, dx = (torch.empty_like(x) for _ in range(4))
    mean, rstd, dgamma, dbeta = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ctx.layer_norm(x, gamma, beta, y, residual=res, total=total, mean=mean, rstd=rstd, mask=spec)
    t, m, r, h, want = norm64(x, res, gamma, beta, 1e-5, mask)
    # rows of normal numbers: |t| below 12, |h| below 8, rstd below 1.1; 64 + cols / 4096 < 82 additions
    close(y, want, 82 * U * 12 * 1.1 * 17 * gamma.double().abs() + 64 * U * want.abs() + rounding(ty, want))
    close(total, t, 4 * U * 12 + rounding(ty, t))
    ctx.layer_norm_gradients(dy, total, mean, rstd, gamma, dr, dgamma=dgamma, dbeta=dbeta, dtotal=x, dx=dx, mask=spec)
    d, wx, wg, wb = back64(dy, total, mean, rstd, gamma, x, mask)
    close(dr, d, 82 * U * 60 + rounding(ty, d))
    close(dx, wx, 82 * U * 80 + rounding(ty, wx))
    close(dgamma, wg.sum(0), 8 * U * 60 * rows)
    close(dbeta, wb.sum(0), 8 * U * 8 * rows)
    out = torch.empty_like(x)
    ctx.dropout(x, out, spec)
    assert torch.equal(out, torch.where(mask[0], (x.float() * mask[1]).to(ty), torch.zeros_like(x)))
    ctx.close()


def test_rows_more_than_two_to_the_31_apart(rt):  # noqa: F811
    ld, rows, cols, n_out = (1 << 30) + 24, 3, 333, 40
    big = torch.empty(2 * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((rows, cols), (ld, 1))
    value = normal(rows, cols).bfloat16()
    ctx = rt.MatrixContext(max(rt.micro_scratch(rows, n_out, cols), rt.layer_norm_scratch(rows, cols)))
    m = rt.MicroWeights(n_out, cols)
    ctx.micro_weights(normal(n_out, cols, seed=1), m)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    spec = rt.Mask(0.3, 4, 2)

    def results(x, far):
        """Everything once from x, and in place where x is far."""
        y, dw, dx = torch.empty((rows, n_out), dtype=torch.bfloat16, device="cuda"), torch.empty((n_out, cols), device="cuda"), torch.empty_like(value)
        ctx.micro_product(x, m, y)
        ctx.micro_gradients(y, x, m, dx, dw)
        out = x if far else torch.empty_like(x)
        ctx.layer_norm(x, None, None, out, mean=mean, rstd=rstd, mask=spec)
        normed = out.clone()
        ctx.layer_norm_gradients(value, out, mean, rstd, None, dresidual=out)
        back = out.clone()
        ctx.dropout(out, out, spec)
        return y, dw, dx, normed, back, out.clone()
    x.copy_(value)
    far = results(x, True)
    for a, b in zip(far, results(value.clone(), False)):
        assert torch.equal(a.nan_to_num(), b.nan_to_num())
    # results written far apart
    far_out = big.as_strided((rows, n_out), (ld, 1))
    y = torch.empty((rows, n_out), dtype=torch.bfloat16, device="cuda")
    ctx.micro_product(value, m, far_out)
    ctx.micro_product(value, m, y)
    assert torch.equal(far_out, y)
    ctx.close()


@pytest.mark.parametrize("cols", [16384, 33001])
def test_more_than_two_to_the_31_values(rt, cols):  # noqa: F811
    rows = (1 << 31) // cols + 40
    ctx = rt.MatrixContext(0)
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-5:] = normal(5, cols).bfloat16()
    y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    spec = rt.Mask(0.25, 6)
    mask = kept(5, cols, 0.25, 6, row0=rows - 5)
    ctx.dropout(x, y, spec)
    assert torch.equal(y[-5:], torch.where(mask[0], (x[-5:].float() * mask[1]).bfloat16(), torch.zeros_like(x[-5:])))
    assert not bool(y[:-5:97].any())
    ctx.layer_norm(x, None, None, y, rstd=rstd, mask=spec)
    _, _, r, _, want = norm64(x[-5:], None, None, None, 1e-5, mask)
    close(y[-5:], want, 82 * U * 12 * 1.1 * 17 + rounding(torch.bfloat16, want))
    close(rstd[-5:], r, 300 * U * r)
    assert not bool(y[:-5:97].any())
    ctx.close()


def test_many_short_rows(rt):  # noqa: F811
    rows, cols = 300001, 9
    x, dy = normal(rows, cols), normal(rows, cols, seed=1)
    ctx = rt.MatrixContext(rt.layer_norm_scratch(rows, cols))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dgamma, dbeta = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ctx.layer_norm(x, None, None, y, mean=mean, rstd=rstd)
    _, _, r, h, want = norm64(x, None, None, None, 1e-5, None)
    close(y, want, 64 * U * (x.double().abs().amax(1) * r)[:, None] * (1 + 2 * h.abs()) + 64 * U * h.abs())
    ctx.layer_norm_gradients(dy, x, mean, rstd, None, dx, dgamma=dgamma, dbeta=dbeta)
    _, _, wg, wb = back64(dy, x, mean, rstd, None, None, None)
    # a block adds at most 300001 / 148 + 16 rows in turn, in groups: 130 additions of 16 groups, then 148 blocks in binary64
    close(dgamma, wg.sum(0), 200 * U * wg.abs().sum(0) + 8 * U * (dy.double().abs() * (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]).sum(0))
    close(dbeta, wb.sum(0), 200 * U * wb.abs().sum(0))
    ctx.close()


def test_no_call_leaves_its_scratch(rt):  # noqa: F811
    """Contexts on the caller's memory of just the size that is asked for, with bytes around it that must stay."""
    lib, stream = rt.load_library(), torch.cuda.current_stream().cuda_stream
    for tokens, n_in, n_out in ((1, 33, 1), (7, 300, 129), (200, 515, 700), (129, 1500, 64)):
        need = max(rt.micro_scratch(tokens, n_out, n_in), rt.layer_norm_scratch(tokens, n_in))
        memory = torch.full((need + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
        handle = ctypes.c_void_p()
        assert lib.rtopk_matrix_create(ctypes.byref(handle), 0, memory.data_ptr() + 4096, need, stream) == 0
        ctx = rt.MatrixContext(0)
        own, ctx._h = ctx._h, handle
        m = rt.MicroWeights(n_out, n_in)
        x, dy, w = normal(tokens, n_in), normal(tokens, n_out, seed=1), normal(n_out, n_in, seed=2)
        ctx.micro_weights(w, m)
        y, dx, dw, v = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty(n_in, device="cuda")
        ctx.micro_product(x, m, y)
        ctx.micro_gradients(dy, x, m, dx, dw)
        ctx.layer_norm_gradients(x, x, x[:, 0].contiguous(), x[:, 0].contiguous(), None, dgamma=v, dbeta=v.clone())
        ctx.poll_status()
        assert bool((memory[:4096] == 0x5A).all()) and bool((memory[4096 + need:] == 0x5A).all())
        ctx.close()
        ctx._h = own
        ctx.close()


def test_codes_stay_inside_their_rows(rt):  # noqa: F811
    """Codes of wider rows than asked for: what is past a whole number of blocks stays."""
    n_out, n_in = 70, 45
    m = rt.MicroWeights(n_out, n_in)
    m.codes, m.codes_t = torch.full((n_out, 64), 0x5A, dtype=torch.uint8, device="cuda"), torch.full((n_in, 96), 0x5A, dtype=torch.uint8, device="cuda")
    ctx = rt.MatrixContext(0)
    w = normal(n_out, n_in)
    ctx.micro_weights(w, m)
    assert bool((m.codes[:, 32:] == 0x5A).all()) and bool((m.codes_t[:, 48:] == 0x5A).all())
    assert not bool(m.codes[:, 23:32].any()) and not bool(m.codes_t[:, 35:48].any())
    assert torch.equal(m.dense().double(), coded(w, 32))
    other = copy.deepcopy(m)
    m.codes.zero_()
    assert torch.equal(other.dense().double(), coded(w, 32))
    ctx.close()


def test_micro_products_that_give_up_leave_no_copy_behind(rt):  # noqa: F811
    """Every tile of the product kernel on 4-bit codes, whole and in parts, behaving as if a wait had run out: each call reports for itself and ends long
    before the limit of a wait (2 s), nothing around the results is written, and what runs right behind it is right."""
    layers = [(30, 300, 200), (300, 500, 400), (100, 8192, 300), (700, 1500, 1500), (1100, 4100, 2000), (4096, 2048, 4096), (60, 70000, 40)]
    ctx = rt.MatrixContext(max(rt.micro_scratch(t, n, k) for t, k, n in layers))

    def calls():
        for t, k, n in layers:
            m = rt.MicroWeights(n, k)
            w, x, dy = normal(n, k, seed=t), normal(t, k, seed=t + 1), normal(t, n, seed=t + 2)
            ctx.micro_weights(w, m)
            y, both = torch.full((t + 2, n + 8), 9.0, device="cuda"), torch.full((t * k + n * k,), 9.0, device="cuda")
            yield lambda: ctx.micro_product(x, m, y[1:1 + t, 8:]), y, y[1:1 + t, 8:]
            dx, dw = both[:t * k].view(t, k), both[t * k:].view(n, k)
            yield lambda: ctx.micro_gradients(dy, None, m, dx=dx), both, dx
            yield lambda: ctx.micro_gradients(dy, x, m, dw=dw), both, dw
            yield lambda: ctx.micro_gradients(dy, x, m, dx, dw), both, both

    for call, around, out in calls():
        around.fill_(9.0)
        call()
        want = out.clone()
        out.fill_(9.0)
        assert bool((around == 9.0).all())
        torch.cuda.synchronize()
        ctx.set_option(0, 1)
        t0 = time.monotonic()
        call()
        with pytest.raises(rt.RTopKError) as e:
            ctx.poll_status()
        assert e.value.status == 5
        assert time.monotonic() - t0 < 1.0
        out.fill_(9.0)
        assert bool((around == 9.0).all())
        call()
        ctx.set_option(0, 0)
        with pytest.raises(rt.RTopKError):
            ctx.poll_status()
        for _ in range(2):
            out.fill_(9.0)
            call()
            assert torch.equal(out, want)
        ctx.poll_status()
    ctx.close()
