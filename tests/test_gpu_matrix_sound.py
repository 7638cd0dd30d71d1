"""The matrix operators where precision, range, lengths and the handling of errors are easily lost.  Definitions and what is not said
here as in test_gpu_matrix.py."""
import pytest
import torch

from test_gpu_matrix import U16, code64, gen, matrices, near, orth64, rel, rt  # noqa: F401

pytestmark = pytest.mark.gpu


def orthogonalize(rt, u, ty=torch.float32, **kw):  # noqa: F811
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(*u.shape))
    out = torch.full(u.shape, 7.0, dtype=ty, device="cuda")
    ctx.orthogonalize(u, out, **kw)
    ctx.poll_status()
    ctx.close()
    return out


def orthogonal_rows(m, n, seed=0):
    """Rows (columns of a tall one) that share no position: the Gram matrix is diagonal."""
    s, l = min(m, n), max(m, n)
    u = torch.zeros((1, s, l), device="cuda")
    j = torch.arange(l, device="cuda")
    u[0, j % s, j] = torch.randn(l, generator=gen(seed), device="cuda")
    return u if m <= n else u.mT.contiguous()


# What orthogonal rows leave is x times a polynomial of the row's own sum of squares, all in 32 bits.  A sum of some hundred squares, taken in two
# levels: errors of 8 x 2^-25 together; the polynomial is up to ten times as sensitive, and five steps let an error grow by
# 1.6 each, ten times: 2.4e-5.  3e-5 taken.  An X that is read from 16 bits alone would be 2^-11 / sqrt(6) = 2e-4 off.
ORTHOGONAL_ROWS = 3e-5


@pytest.mark.parametrize("m,n", [(200, 1000), (1000, 200), (60, 200), (100, 1000), (512, 4000), (131, 133)])
def test_x_stays_in_32_bits_to_the_result(rt, m, n):  # noqa: F811
    u = orthogonal_rows(m, n)
    for steps in (1, 2, 5):
        assert rel(orthogonalize(rt, u, steps=steps), orth64(u, steps)) <= ORTHOGONAL_ROWS, steps
    g, v, w = u * 1e-3, torch.zeros_like(u), torch.zeros_like(u)
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(1, m, n))
    ctx.orthogonal_update(g, v, w, 1.0, 0.5, scale=-1.0)
    assert rel(w, orth64(g + 0.5 * g)) <= ORTHOGONAL_ROWS
    ctx.close()


def test_products_that_give_up_leave_no_copy_behind(rt):  # noqa: F811
    """Blocks and pairs of blocks of the product kernel, with few steps (all copies issued, none waited for by the feeding warp) and
    with many, the pair's blocks at different steps when they stop.  Every call reports for itself; it ends long before the
    limit of a wait (2 s), so the copies in flight were waited for and not timed out; what runs right behind it is right."""
    import time
    shapes = [(200, 1500), (300, 300), (1300, 1400), (2100, 700)]
    layers = [(300, 500, 400), (64, 600, 300), (1100, 4100, 2000), (2000, 200, 1500)]
    ctx = rt.MatrixContext(max([rt.orthogonalize_scratch(1, a, b) for a, b in shapes] + [rt.coded_scratch(t, n, k) for t, k, n in layers]))

    def calls():
        for a, b in shapes:
            u, out = torch.randn((a, b), generator=gen(a), device="cuda"), torch.empty((a, b), device="cuda")
            yield lambda: ctx.orthogonalize(u, out), out
            v, w = torch.zeros_like(u), torch.zeros_like(u)
            yield lambda: (v.zero_(), w.zero_(), ctx.orthogonal_update(u, v, w, 0.1, 0.9)), w
        for t, k, n in layers:
            coded = rt.CodedWeights(n, k)
            w, x, dy = (torch.randn(s, generator=gen(t), device="cuda") for s in ((n, k), (t, k), (t, n)))
            ctx.code_weights(w, coded)
            y, dx, dw = torch.empty((t, n), device="cuda"), torch.empty((t, k), device="cuda"), torch.empty((n, k), device="cuda")
            yield lambda: ctx.coded_product(x, coded, y), y
            yield lambda: ctx.coded_gradients(dy, None, coded, dx=dx), dx
            yield lambda: ctx.coded_gradients(dy, x, coded, dw=dw), dw
            both = torch.empty((t * k + n * k,), device="cuda")
            yield lambda: ctx.coded_gradients(dy, x, coded, both[:t * k].view(t, k), both[t * k:].view(n, k)), both

    for call, out in calls():
        call()
        want = out.clone()
        torch.cuda.synchronize()
        ctx.set_option(0, 1)
        t0 = time.monotonic()
        call()
        with pytest.raises(rt.RTopKError) as e:
            ctx.poll_status()
        assert e.value.status == 5
        assert time.monotonic() - t0 < 1.0
        call()
        ctx.set_option(0, 0)
        with pytest.raises(rt.RTopKError):      # clears the counters of parts that were never added up
            ctx.poll_status()
        for _ in range(2):
            out.fill_(9.0)
            call()
            assert torch.equal(out, want)
        ctx.poll_status()
    ctx.close()


def test_coded_weights_received_copied_and_moved(rt):  # noqa: F811
    """The calls read and write the tensors that the object holds at the time."""
    import copy
    t, k, n = 5, 200, 96
    ctx = rt.MatrixContext(rt.coded_scratch(t, n, k))
    a, b = rt.CodedWeights(n, k), rt.CodedWeights(n, k)
    wa, wb, x = (torch.randn(s, generator=gen(i), device="cuda") for i, s in enumerate(((n, k), (n, k), (t, k))))
    ctx.code_weights(wa, a)
    ctx.code_weights(wb, b)

    def product(c):
        y, dx = torch.empty((t, n), device="cuda"), torch.empty((t, k), device="cuda")
        ctx.coded_product(x, c, y)
        ctx.coded_gradients(y, None, c, dx=dx)
        return y, dx

    def same(p, q):
        return all(torch.equal(u, v) for u, v in zip(p, q))
    of_a, of_b = product(a), product(b)
    assert not same(of_a, of_b)
    received = rt.CodedWeights(n, k)
    received.codes, received.codes_t, received.scales = (v.clone() for v in (b.codes, b.codes_t, b.scales))
    assert same(product(received), of_b)
    copied = copy.deepcopy(a)
    ctx.code_weights(wb, copied)                    # the original keeps its codes
    assert same(product(copied), of_b) and same(product(a), of_a)
    ctx.close()


def test_more_rows_than_32_bits_of_threads(rt):  # noqa: F811
    """Eight rows a block of 256 threads: past 2^26 rows a thread's number in the launch no longer fits 31 bits.  Rows are compared at
    both ends and around that one."""
    n, k, m = (1 << 26) + 41, 8, 3
    at = torch.cat([torch.arange(64), torch.arange((1 << 26) - 32, (1 << 26) + 41)]).cuda()
    x = torch.empty((n, k), dtype=torch.bfloat16, device="cuda").normal_(generator=gen(1))
    coded = rt.CodedWeights(n, k, transposed=False)
    ctx = rt.MatrixContext(0)
    ctx.code_weights(x, coded)
    q, s = code64(x[at], 1)
    assert torch.equal(coded.codes[at][:, :k].double(), q) and torch.equal(coded.scales[at].double(), s.flatten())
    assert bool((coded.scales > 0).all())
    ctx.close()
    del coded
    w = torch.randn((m, k), generator=gen(2), device="cuda")
    ctx, coded = rt.MatrixContext(rt.coded_scratch(n, m, k)), rt.CodedWeights(m, k)
    ctx.code_weights(w, coded)
    out = torch.full((n, m), float("nan"), dtype=torch.bfloat16, device="cuda")
    ctx.coded_product(x, coded, out)
    ctx.poll_status()
    qw, sw = code64(w, 1)
    near(out[at], (q @ qw.t()) * s * sw.t(), torch.bfloat16)
    assert not bool(out.isnan().any())             # every row was written
    ctx.close()


@pytest.mark.parametrize("m,n", [(40, 96), (96, 40), (100, 700), (200, 300), (300, 200)])
def test_norms_at_both_ends_of_the_range(rt, m, n):  # noqa: F811
    """The whole range of binary32: with eps = 0 entries down to single steps of the subnormal numbers, where 1 / norm is past the range,
    and entries near the largest number, where it is subnormal."""
    u = matrices("gauss", 1, m, n, 6)
    for scale in (1e-36, 1e-38, 1e-39, 1e-41, 1e-44):
        v = u * scale
        want = orth64(v, eps=0.0)
        assert rel(orthogonalize(rt, v, eps=0.0), want) <= 4 * U16, scale
        zeros = v.clone()
        zeros[:, 0] = 0.0                           # zero times an infinite factor would be NaN
        assert rel(orthogonalize(rt, zeros, eps=0.0), orth64(zeros, eps=0.0)) <= 4 * U16, scale
        g, mom, w = v.clone(), torch.zeros_like(v), torch.zeros_like(v)
        ctx = rt.MatrixContext(rt.orthogonalize_scratch(1, m, n))
        ctx.orthogonal_update(g, mom, w, 1.0, 0.0, scale=-1.0, eps=0.0)
        assert torch.equal(mom, v) and rel(w, want) <= 4 * U16, scale
        ctx.close()
    big = u / u.abs().max() * 3.4e38
    assert rel(orthogonalize(rt, big), orth64(big)) <= 4 * U16
    full = torch.full_like(u, 3.4e38) * torch.sign(u)
    assert rel(orthogonalize(rt, full), orth64(full)) <= 4 * U16


def test_no_tokens_need_no_scratch(rt):  # noqa: F811
    ctx, coded = rt.MatrixContext(0), rt.CodedWeights(40, 30)
    f = lambda *s: torch.full(s, 2.0, device="cuda")       # noqa: E731
    dw = f(40, 33)
    ctx.coded_product(f(0, 30), coded, f(0, 40))
    ctx.coded_gradients(f(0, 40), f(0, 30), coded, f(0, 30), dw[:, :30])
    ctx.poll_status()
    assert bool((dw[:, :30] == 0).all()) and bool((dw[:, 30:] == 2.0).all())
    with pytest.raises(rt.RTopKError):                      # arguments are looked at all the same
        ctx.coded_gradients(f(0, 40), f(0, 30), coded)
    ctx.close()


@pytest.mark.parametrize("n", [1 << 16, (1 << 22) + 8, 1 << 25])
def test_long_rows_of_equal_squares(rt, n):  # noqa: F811
    """Equal terms make every rounding of a chain of sums fall the same way.  One row has no products, only its sum of squares: the bound is
    that of orthogonal rows."""
    for u in (torch.ones((1, 1, n), device="cuda"), torch.full((1, min(n, 64 * 65535), 1), -0.3, device="cuda")):      # as many rows as are taken
        assert rel(orthogonalize(rt, u), orth64(u)) <= ORTHOGONAL_ROWS


@pytest.mark.parametrize("n", [1 << 12, 1 << 17, (1 << 20) + 24, 1 << 22, 1 << 24])
def test_long_rows_that_nearly_depend_on_each_other(rt, n):  # noqa: F811
    """What the tensor core adds up in one accumulator loses a little at every step, always downwards; the products of nearly equal rows
    show it most.  One step of two rows has one entry off each diagonal, about 0.5 of a Gram matrix with an eigenvalue near 1 and
    a + b + c = 0.70 times X as the result.  Rounding that entry to 16 bits (u = 2^-11 of it) moves the result by |b + 2 c| 0.5 u = 0.36 u;
    the polynomial's, (b + c) 0.5 = -1.37, by 1.37 u: 2.5 u of 0.70 together.  3 u taken, whatever the length."""
    u = matrices("gauss", 1, 2, n)
    u[0, 1] = u[0, 0] + 0.1 * u[0, 1]
    t = torch.ones((1, 2, n), device="cuda")
    t[0, 1, ::2] = 0.5
    for v in (u, t, t[:, :, :min(n, 64 * 65535)].mT.contiguous()):
        assert rel(orthogonalize(rt, v, steps=1), orth64(v, 1)) <= 3 * U16


@pytest.mark.parametrize("m,n", [(60, 200), (100, 1500), (300, 700)])
def test_many_steps(rt, m, n):  # noqa: F811
    """The default step has slopes of up to -1.6 where it keeps the singular values, so an error grows with the steps instead of
    shrinking; it ends at some percent because the values stay in a band.  Measured for 300 x 700 2.3e-3 after 16 steps and 9.1e-3 after 64, less in
    the smaller ones; twice that is taken.  The cubic step has slope 0 at 1: its last steps' roundings alone are left, 4 u."""
    u = matrices("gauss", 1, m, n)
    for steps, most in ((16, 4.6e-3), (64, 1.8e-2)):
        assert rel(orthogonalize(rt, u, steps=steps), orth64(u, steps)) <= most, steps
        cubic = [(1.5, -0.5, 0.0)] * steps
        assert rel(orthogonalize(rt, u, steps=steps, coef=cubic), orth64(u, steps, coef=cubic)) <= 4 * U16, steps


def test_a_context_used_on_another_stream_than_it_was_made_on(rt):  # noqa: F811
    """Its scratch comes from torch's allocator, which hands out memory that the making stream may still be using; a call on another stream
    must not write there before that stream is done with it."""
    t, k, n = 200, 300, 1200
    size = rt.coded_scratch(t, n, k)
    coded, x, y = rt.CodedWeights(n, k), torch.randn((t, k), generator=gen(1), device="cuda"), torch.empty((t, n), device="cuda")
    ctx = rt.MatrixContext(size)
    ctx.code_weights(torch.randn((n, k), generator=gen(2), device="cuda"), coded)
    ctx.coded_product(x, coded, y)
    want = y.clone()
    ctx.close()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    old = torch.ones(size, dtype=torch.uint8, device="cuda")
    at = old.data_ptr()
    assert int(old.sum()) == size                   # its kernel is loaded from here on
    torch.cuda.synchronize()
    torch.cuda._sleep(300_000_000)                  # 0.15 s, no more than one block
    total = old.sum()
    del old
    ctx = rt.MatrixContext(size)
    assert ctx._scratch.data_ptr() == at            # the case in question
    with torch.cuda.stream(side):
        y.zero_()
        ctx.coded_product(x, coded, y)
    torch.cuda.synchronize()
    assert int(total) == size
    assert torch.equal(y, want)
    # and captured on a stream of its own
    graph = torch.cuda.CUDAGraph()
    ctx = rt.MatrixContext(size)
    with torch.cuda.graph(graph):
        ctx.coded_product(x, coded, y)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    ctx.poll_status()
    ctx.close()
