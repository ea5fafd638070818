"""Orthogonalised updates of stacks that are computed in tiles of 128, through several steps along
the summed axis, against the 64-bit iteration, value by value."""
import pytest
import torch

from encoder_reference import UNIT, check
from test_gpu_orth import DTYPES, FIVE, _matrices, ps  # noqa: F401
from training_reference import near, orthogonalize_bound

pytestmark = pytest.mark.gpu


def _last_step(g):
    """Of the last of five steps, the products of magnitudes that enter each value: of B with X,
    and of A, C and X in B = a I + A C."""
    a, b, c = FIVE
    x = g.double()
    x = x / (x.square().sum().sqrt() + 1e-7)
    x = x if x.shape[0] <= x.shape[1] else x.T
    eye = torch.eye(x.shape[0], dtype=torch.float64)
    for _ in range(5):
        gram = x @ x.T
        poly = a * eye + gram @ (b * eye + c * gram)
        size = poly.abs() @ x.abs(), gram.abs() @ (b * eye + c * gram).abs() @ x.abs()
        x = poly @ x
    return size if g.shape[0] <= g.shape[1] else tuple(s.T for s in size)


@pytest.mark.parametrize("batch, m, n", [(24, 300, 520), (24, 517, 301), (23, 384, 384),
                                         (130, 100, 72)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_orthogonalize_stacks(ps, batch, m, n, dtype):  # noqa: F811
    tiles = -(-min(m, n) // 128)
    assert tiles * (tiles + 1) // 2 * batch > 128  # of the launch that has fewest
    g = _matrices(batch, m, n, m + 3 * n).to(DTYPES[dtype])
    u = UNIT[DTYPES[dtype]]
    got = ps.orthogonalize(g.cuda())
    for i in range(batch):
        val, bound = orthogonalize_bound(g[i], 5, FIVE, 1e-7)
        near(f"matrix {i}", got[i], val, bound)
        # no value is off by more than the whole matrix may be, and its own rounding; in bfloat16
        # the last step's factors have 11 bits each (off by 2^-11)
        off = (bound - (u if dtype != "f32" else 0.0)) * float(val.norm())
        tol = u * val.abs() + off
        if dtype == "bf16":
            bx, acx = _last_step(g[i])
            tol = tol + 2 * 2.0 ** -11 * (bx + acx)
        check(f"matrix {i}", got[i], val, (1 + u) * tol)
    assert torch.equal(got, ps.orthogonalize(g.cuda()))
