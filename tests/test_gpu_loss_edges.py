"""Cross entropy where finite inputs go wrong first."""
import math

import pytest
import torch

from encoder_reference import check
from test_gpu_loss import DTYPES, _inputs, _rnd, _run, ps  # noqa: F401
from training_reference import cross_entropy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("large", [30.0, 64.0, 110.0])
def test_loss_of_channels_that_cancel(ps, dtype, large):  # noqa: F811
    """Two channels far larger than the others, whose products cancel: a logit's rounding error is
    then well above its row's 1 - p, of about 0.001, and gradients stay finite and within it."""
    g, rnd = _rnd(21)
    rows, vocab, n = 600, 300, 768
    targets = torch.randint(vocab, (rows,), generator=g)
    table = rnd(vocab, n) * n ** -0.5
    h = rnd(rows, n) + (11 + 5 * torch.rand(rows, 1, generator=g)) * table[targets]
    table[:, 100], table[:, 600] = large, -large
    h[:, 100] = h[:, 600] = large
    h, table = h.to(DTYPES[dtype]), table.to(DTYPES[dtype])
    dloss = torch.full((rows,), 1.0 / rows)
    val, tol = cross_entropy(h, table, targets, 1.0, dloss)
    got = _run(ps, h, table, targets, dloss)
    for name in val:
        assert got[name].isfinite().all(), name
        check(name, got[name], val[name], tol[name])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_loss_of_rows_that_are_not_numbers_in_any_type(ps, dtype, bad):  # noqa: F811
    """They stay that: nothing that keeps finite values in range makes numbers of them."""
    h, table, targets, dloss = _inputs(70, 300, 40, DTYPES[dtype], 5, left_out=0.0)
    h[3, 7] = bad
    got = _run(ps, h, table, targets, dloss)
    rest = (torch.arange(70) != 3).cuda()
    assert not got["lse"][3].isfinite() and got["lse"][rest].isfinite().all()
    assert not got["dh"][3].isfinite().any() and got["dh"][rest].isfinite().all()
    assert not got["dtable"].isfinite().any()
    table[5, 7] = math.nan
    got = _run(ps, h, table, targets, dloss)
    for name in ("loss", "lse", "dh", "dtable"):
        assert got[name].isnan().all(), name
