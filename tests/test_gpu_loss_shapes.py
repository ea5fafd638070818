"""Cross entropy at sizes that take each shape of the tiles through several steps and several tiles
a work-group, and each loop around the launches twice: value by value against the 64-bit oracle,
which runs on the GPU here for its size."""
import pytest
import torch

from encoder_reference import check
from test_gpu_loss import DTYPES, RMS, _inputs, _run, ps  # noqa: F401
from training_reference import cross_entropy, near

pytestmark = pytest.mark.gpu

#: rows, vocab, n, types, and what the rules choose: the tiles of the forward pass, of g and of the
#: products, the planes of weighed h, the pieces of the vocabulary in the backward pass
SHAPES = [
    (500, 16001, 515, ("f16", "bf16"), "small", "small", "small", 1, 1),
    (700, 9001, 515, ("f16", "bf16"), "small", "small", "deep", 1, 1),
    (300, 12001, 515, ("f16", "bf16"), "small", "small", "large", 2, 1),
    (2600, 20100, 515, ("f16", "bf16"), "large", "large", "large", 1, 1),
    (5000, 40001, 136, ("f16", "bf16"), "large", "large", "large", 1, 2),
    (3000, 9001, 136, ("f32",), "triple", "triple", "triple", 3, 1),
    # more rows than a launch of the forward pass takes
    (66000, 300, 72, ("f16",), "large", "large", "deep", 2, 1),
    (66000, 2100, 72, ("bf16",), "large", "large", "deep", 1, 2),
    (66000, 2100, 72, ("f32",), "triple", "triple", "triple", 3, 5),
    # more vectors than a launch takes of a table that is read where it lies
    (20, (1 << 20) + 3001, 8, ("bf16",), "small", "small", "deep", 2, 17),
]


def _against_oracle(ps, rows, vocab, n, dtype):  # noqa: F811
    x = _inputs(rows, vocab, n, DTYPES[dtype], rows + 3 * n)
    got = _run(ps, *x)
    c = [t.cuda() for t in x]
    val, tol = cross_entropy(*c[:3], 1.0, c[3])
    for name in val:
        check(name, got[name], val[name].cpu(), tol[name].cpu())
    for name in ("dh", "dtable"):
        want = val[name].cpu()
        # gradients of a mean over many rows lie below binary16's normal range (2^-14), where a
        # rounding is off by up to 2^-25 whatever the value is
        step = 2.0 ** -25 * want.numel() ** 0.5 if dtype == "f16" else 0.0
        near(name, got[name], want, RMS[dtype] + step / float(want.norm()))
    again = _run(ps, *x)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("rows, vocab, n, dtype",
                         [s[:3] + (d,) for s in SHAPES for d in s[3]])
def test_loss_shapes(ps, rows, vocab, n, dtype):  # noqa: F811
    _against_oracle(ps, rows, vocab, n, dtype)


@pytest.mark.parametrize("rows, dtype", [(1, "f16"), (3, "bf16"), (4, "f16"), (1, "f32"),
                                         (16, "f32")])
@pytest.mark.parametrize("vocab", [70001, 200003])
def test_loss_of_few_rows_and_many_vectors(ps, rows, dtype, vocab):  # noqa: F811
    """Rows straight from the table, where a work-group takes several groups of vectors."""
    h, table, targets, _ = _inputs(rows, vocab, 72, DTYPES[dtype], rows + 5, left_out=0.0)
    loss, lse = ps.linear_cross_entropy_forward(h.cuda(), table.cuda(), targets.cuda())
    val, tol = cross_entropy(h, table, targets, 1.0)
    check("loss", loss, val["loss"], tol["loss"])
    check("lse", lse, val["lse"], tol["lse"])
