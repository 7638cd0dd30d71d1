"""The matrix operators where precision, range, lengths and the handling of errors are easily lost.  Definitions and what is not said
here as in test_gpu_matrix.py."""
import pytest
import torch

from test_gpu_matrix import U16, gen, mu_exact, orth64, rel, rt  # noqa: F401

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
