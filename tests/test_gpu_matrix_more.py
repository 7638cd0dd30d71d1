"""The matrix operators where their kernels change: shapes on both sides of every choice, views far apart in memory, the loop that
uses them together.  Tolerances as derived in test_gpu_matrix.py."""
import os
import sys

import pytest
import torch

from test_gpu_matrix import U16, code64, matrices, mu_exact, near, orth64, rel, rt, tokens_of  # noqa: F401

pytestmark = pytest.mark.gpu

# one block, clusters of two to eight, just past them; tall, wide, batched
EDGES = [(1, 64, 256), (1, 64, 257), (1, 65, 65), (1, 128, 128), (2, 128, 257), (3, 100, 513), (1, 128, 1025), (1, 90, 2048), (1, 2048, 90), (2, 128, 2049),
         (1, 129, 300), (1, 300, 129), (20, 128, 300), (1, 3, 2000), (1, 512, 512), (2, 1500, 512), (1, 256, 4100)]


@pytest.mark.parametrize("batch,m,n", EDGES)
def test_orthogonalize_at_the_edges(rt, batch, m, n):  # noqa: F811
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(batch, m, n))
    for kind in ("gauss", "low"):
        u = matrices(kind, batch, m, n, 5)
        out = torch.full((batch, m, n), 7.0, device="cuda")
        ctx.orthogonalize(u, out)
        ctx.poll_status()
        want = orth64(u)
        for z in range(batch):
            assert rel(out[z], want[z]) <= 4 * U16, (kind, z)
    ctx.close()


@pytest.mark.parametrize("m,n", [(100, 700), (700, 100), (128, 200), (130, 600)])
def test_orthogonal_update_at_the_edges(rt, m, n):  # noqa: F811
    ctx = rt.MatrixContext(rt.orthogonalize_scratch(2, m, n))
    g, v, w = (matrices(k, 2, m, n, i) * s for i, (k, s) in enumerate((("sparse", 1e-3), ("low", 1e-3), ("gauss", 0.05))))
    big = torch.zeros((2, m, n + 3), device="cuda")
    mom = big[..., 1:1 + n]                       # rows that allow no vector loads
    mom.copy_(v)
    weights = w.clone()
    ctx.orthogonal_update(g, mom, weights, 0.02, 0.9, decay=0.1, scale=3.0)
    v64 = mu_exact(0.9) * v.double() + g.double()
    assert float((mom.double() - v64).abs().max() / (v64.abs() + g.abs().double()).max()) <= 2.0 ** -23
    o = orth64(g.double() + mu_exact(0.9) * mom.double())
    want = w.double() * (1 - 0.02 * 0.1) - 0.02 * 3.0 * o
    for z in range(2):
        assert float((weights[z].double() - want[z]).norm()) <= 3 * 2.0 ** -24 * float(want[z].norm()) + 0.02 * 3.0 * 4 * U16 * float(o[z].norm())
    assert bool((big[..., 0] == 0).all()) and bool((big[..., 1 + n:] == 0).all())
    ctx.close()


def test_matrices_more_than_two_to_the_31_apart(rt):  # noqa: F811
    m, n, far = 200, 300, (1 << 31) + 72
    base = torch.empty(far + m * n, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(far + m * n, dtype=torch.bfloat16, device="cuda")
    src, dst = (t.as_strided((2, m, n), (far, n, 1)) for t in (base, out))
    src.copy_(matrices("gauss", 2, m, n).bfloat16())
    ctx = rt.MatrixContext(max(rt.orthogonalize_scratch(2, m, n), rt.coded_scratch(20, m, n)))
    ctx.orthogonalize(src, dst)
    want = orth64(src)
    for z in range(2):
        assert rel(dst[z], want[z]) <= 4 * U16 + 2.0 ** -8
    # two, and twenty, tokens whose rows are that far apart
    coded = rt.CodedWeights(m, n)
    w = tokens_of(m, n, 1, torch.float32)
    ctx.code_weights(w, coded)
    qw, sw = code64(w, 1)
    x, y = (t.as_strided((2, k), (far, 1)) for t, k in ((base, n), (out, m)))
    ctx.coded_product(x, coded, y)
    qx, sx = code64(x, 1)
    near(y, (qx @ qw.t()) * sx * sw.t(), torch.bfloat16)
    dx, dw = torch.empty((2, n), dtype=torch.bfloat16, device="cuda"), torch.empty((m, n), device="cuda")
    ctx.coded_gradients(y, x, coded, dx, dw)
    qy, sy = code64(y, 0)
    qx, sx = code64(x, 0)
    near(dw, (qy.t() @ qx) * sy.t() * sx, torch.float32)
    ctx.close()


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("n_in,n_out", [(64, 32), (63, 33), (65, 31), (512, 2000), (4099, 4000), (12000, 50), (20000, 500)])
def test_coded_product_of_few_tokens(rt, tokens, n_in, n_out):  # noqa: F811
    """One launch, integer matrix instructions and the product kernel meet here."""
    ctx = rt.MatrixContext(rt.coded_scratch(tokens, n_out, n_in))
    w, x = tokens_of(n_out, n_in, 1, torch.float32), tokens_of(tokens, n_in, 2, torch.bfloat16)
    coded = rt.CodedWeights(n_out, n_in, transposed=False)
    coded.codes.fill_(99)                          # what lies past the rows' ends must not count
    ctx.code_weights(w, coded)
    out = torch.zeros((tokens, n_out), dtype=torch.bfloat16, device="cuda")
    ctx.coded_product(x, coded, out)
    qx, sx = code64(x, 1)
    qw, sw = code64(w, 1)
    near(out, (qx @ qw.t()) * sx * sw.t(), torch.bfloat16)
    assert n_in == coded.codes.shape[1] or bool((coded.codes[:, n_in:] == 99).all())
    ctx.close()


def test_codes_of_exact_middles_go_to_even(rt):  # noqa: F811
    """max = 127 gives s = 1: every quotient is the value itself, and halves go to the even neighbour."""
    v = torch.arange(-254, 255, device="cuda").float() / 2
    w = torch.stack([v, v.flip(0), v * 2.0 ** -140])          # the last among the subnormal numbers
    coded = rt.CodedWeights(3, v.numel())
    ctx = rt.MatrixContext(0)
    ctx.code_weights(w, coded)
    q, s = code64(w, 1)
    assert torch.equal(coded.codes[:, :v.numel()].double(), q) and torch.equal(coded.scales.double(), s.flatten())
    assert torch.equal(coded.codes[0, :v.numel()].float(), v.round())
    ctx.close()


def test_a_context_on_the_library_s_own_scratch(rt):  # noqa: F811
    """Through the C interface with scratch = null; a context that is too small refuses and writes nothing."""
    import ctypes as C
    lib, h, m, n = rt.load_library(), C.c_void_p(), 300, 400
    assert lib.rtopk_matrix_create(C.byref(h), 0, None, rt.orthogonalize_scratch(1, m, n), None) == 0
    u = matrices("gauss", 1, m, n)[0]
    out = torch.zeros_like(u)
    torch.cuda.synchronize()
    call = lambda mm: lib.rtopk_orthogonalize(h, u.data_ptr(), 0, n, 0, out.data_ptr(), 0, n, 0, 1, mm, n, 5, None, 1e-7, None)  # noqa: E731
    assert call(m) == 0 and lib.rtopk_matrix_poll_status(h, None) == 0
    assert rel(out, orth64(u)) <= 4 * U16
    assert lib.rtopk_matrix_destroy(h) == 0
    assert lib.rtopk_matrix_create(C.byref(h), 0, u.data_ptr() + 4, 1024, None) == 1          # misaligned
    assert lib.rtopk_matrix_create(C.byref(h), 0, None, -1, None) == 1 and not h.value
    assert lib.rtopk_matrix_create(None, 0, None, 0, None) == 1


def test_the_round_of_the_example_learns():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    try:
        import coded_round
    finally:
        sys.path.pop(0)
    losses = coded_round.train(rounds=60)
    assert all(v == v for v in losses)
    # a fit of the teacher, not its variance: the loss of predicting nothing is the starting loss's order
    assert losses[-1] < 0.35 * losses[0], (losses[0], losses[-1])
    again = coded_round.train(rounds=5)
    assert again == losses[:5]                     # every kernel gives the same bits every time


def test_blocks_that_give_up_say_so_and_leave_everything_in_order(rt):  # noqa: F811
    """Every kernel with waits: one block, a cluster, the chain, products whole and in parts.  What lies around the results stays,
    the status says INTERNAL once, and the next call on the same context is right."""
    shapes = [(60, 60), (100, 900), (200, 1500)]
    t, k, n = 300, 500, 400
    ctx = rt.MatrixContext(max([rt.orthogonalize_scratch(1, a, b) for a, b in shapes] + [rt.coded_scratch(t, n, k)]))
    coded = rt.CodedWeights(n, k)
    w, x = tokens_of(n, k, 1, torch.float32), tokens_of(t, k, 2, torch.float32)
    ctx.code_weights(w, coded)
    for on in (1, 0):
        ctx.set_option(0, on)
        for a, b in shapes:
            u = matrices("gauss", 1, a, b)[0]
            out = torch.full((a + 2, b + 6), 9.0, device="cuda")
            ctx.orthogonalize(u, out[1:1 + a, 3:3 + b])
            got = out[1:1 + a, 3:3 + b].clone()
            out[1:1 + a, 3:3 + b] = 9.0
            assert bool((out == 9.0).all())
            if on:
                with pytest.raises(rt.RTopKError) as e:
                    ctx.poll_status()
                assert e.value.status == 5
            else:
                ctx.poll_status()
                assert rel(got, orth64(u)) <= 4 * U16
        y = torch.full((t + 2, n + 6), 9.0, device="cuda")
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        ctx.coded_product(x, coded, y[1:1 + t, 3:3 + n])
        got = y[1:1 + t, 3:3 + n].clone()
        y[1:1 + t, 3:3 + n] = 9.0
        assert bool((y == 9.0).all())
        ctx.coded_gradients(got, x, coded, dx, dw)
        if on:
            with pytest.raises(rt.RTopKError) as e:
                ctx.poll_status()
            assert e.value.status == 5
            ctx.poll_status()
        else:
            ctx.poll_status()
            qx, sx = code64(x, 1)
            qw, sw = code64(w, 1)
            near(got, (qx @ qw.t()) * sx * sw.t(), torch.float32)
            qy, sy = code64(got, 0)
            qx, sx = code64(x, 0)
            near(dw, (qy.t() @ qx) * sy.t() * sx, torch.float32)
    with pytest.raises(rt.RTopKError):
        ctx.set_option(0, 2)
    ctx.close()


def test_each_call_alone_in_a_graph(rt):  # noqa: F811
    """Calls that begin with a memory set, with a kernel, with another call's kernels just before: captured and replayed."""
    t, k, n = 150, 260, 190
    ctx = rt.MatrixContext(max(rt.coded_scratch(t, n, k), rt.orthogonalize_scratch(1, 100, 900)))
    coded = rt.CodedWeights(n, k)
    w, x, dy = tokens_of(n, k, 1, torch.float32), tokens_of(t, k, 2, torch.float32), tokens_of(t, n, 3, torch.float32)
    u = matrices("gauss", 1, 100, 900)[0]
    ctx.code_weights(w, coded)
    calls = {"dw": lambda o: ctx.coded_gradients(dy, x, coded, dw=o), "dx": lambda o: ctx.coded_gradients(dy, None, coded, dx=o),
             "y": lambda o: ctx.coded_product(x, coded, o), "few": lambda o: ctx.coded_product(x[:2], coded, o), "orth": lambda o: ctx.orthogonalize(u, o)}
    shapes = {"dw": (n, k), "dx": (t, k), "y": (t, n), "few": (2, n), "orth": (100, 900)}
    for name, call in calls.items():
        want, got = torch.zeros(shapes[name], device="cuda"), torch.zeros(shapes[name], device="cuda")
        call(want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(got)
        for _ in range(2):
            got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want), name
    ctx.poll_status()
    ctx.close()


def test_calls_that_share_tensors_one_after_another(rt):  # noqa: F811
    """Launches may start while their predecessors end: results that the next call reads, and inputs that it overwrites."""
    m, n, t = 384, 640, 200
    ctx = rt.MatrixContext(max(rt.orthogonalize_scratch(1, m, n), rt.coded_scratch(t, m, n)))
    coded = rt.CodedWeights(m, n)
    x = tokens_of(t, n, 2, torch.float32)
    w0 = matrices("gauss", 1, m, n)[0] * 0.05

    def chain(sync):
        w, v, g = w0.clone(), torch.zeros_like(w0), torch.zeros_like(w0)
        y, dx = torch.zeros((t, m), device="cuda"), torch.zeros_like(x)
        for _ in range(8):
            ctx.code_weights(w, coded)
            if sync:
                torch.cuda.synchronize()
            ctx.coded_product(x, coded, y)
            if sync:
                torch.cuda.synchronize()
            ctx.coded_gradients(y, x, coded, dx, g)
            if sync:
                torch.cuda.synchronize()
            ctx.orthogonal_update(g, v, w, 0.02, 0.9)
            if sync:
                torch.cuda.synchronize()
        return w, v, y, dx
    want = chain(True)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(chain(False), want))
    ctx.close()
