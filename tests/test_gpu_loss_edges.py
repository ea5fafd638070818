"""Cross entropy where finite inputs go wrong first."""
import math

import pytest
import torch

from encoder_reference import E, UNIT, check
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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 40])
def test_loss_that_is_infinite(ps, dtype, rows):  # noqa: F811
    """A target whose logit lies below fp32's range: its loss is infinite, and the row's gradients
    are those of a probability of 0."""
    h, table, targets, dloss = _inputs(rows, 200, 64, DTYPES[dtype], 22, left_out=0.0)
    t = int(targets[0])
    table[:, 0], h[:, 0] = 0.0, 0.0
    h[0, 0], table[t, 0] = 2.0 ** 66, -2.0 ** 66
    got = _run(ps, h, table, targets, dloss)
    # a logit of some -256 has no probability either, and the first column of dh, which no other
    # vector has a part in, is then 2^124 times smaller
    near_ = table.clone()
    near_[t, 0] = -2.0 ** -58
    val, tol = cross_entropy(h, near_, targets, 1.0, dloss)
    val["loss"][0] = math.inf
    val["dh"][:, 0] *= 2.0 ** 124
    tol["dh"][:, 0] *= 2.0 ** 124
    for name in val:
        check(name, got[name], val[name], tol[name])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("scale", [1.0, 1000.0, 2.0 ** 14])
def test_loss_of_logits_far_apart(ps, dtype, scale):  # noqa: F811
    """Whole numbers, whose logits are exact in fp32: with all others at least 64 below a row's
    largest logit, its gradient is that of the difference of two vectors."""
    g, rnd = _rnd(23)
    h = torch.randint(-3, 4, (50, 16), generator=g).float()
    table = torch.randint(-3, 4, (90, 16), generator=g).float() * 64
    dot = h @ table.t()
    top = dot.argmax(1)
    targets = torch.randint(90, (50,), generator=g)
    only = ((dot == dot.max(1, keepdim=True).values).sum(1) == 1) & (targets != top)
    assert int(only.sum()) > 40
    dt = DTYPES[dtype]
    dloss = torch.full((50,), 1 / scale)
    got = _run(ps, h.to(dt), table.to(dt), torch.where(only, targets, -100), dloss, scale)
    c = only[:, None].double() * scale * float(dloss[0])
    # an exponential is good to 2^-20, g is rounded to dt, and so is the gradient
    off = UNIT[dt] + 2.0 ** -19
    a, b = table[top].double() * c, table[targets].double() * c
    check("dh", got["dh"], a - b, UNIT[dt] * (a - b).abs() + off * (a.abs() + b.abs()) + 1e-20)
    want, size = torch.zeros(90, 16).double(), torch.zeros(90, 16).double()
    for to, sign in ((top, 1), (targets, -1)):
        want.index_add_(0, to, sign * h.double() * c)
        size.index_add_(0, to, h.double().abs() * c)
    # h times its row's factor is rounded, too
    check("dtable", got["dtable"], want, (UNIT[dt] + off) * size + UNIT[dt] * want.abs() + 1e-20)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("power", [17, 19, 20, 21, 22])
def test_loss_of_logits_past_any_use(ps, dtype, power):  # noqa: F811
    """Logits of 2^28 to 2^34: a row's gradient is right, or it is not a number."""
    g, rnd = _rnd(25)
    h = torch.randint(-3, 4, (80, 16), generator=g).float()
    table = torch.randint(-3, 4, (90, 16), generator=g).float() * 64
    dot = h @ table.t()
    top = dot.argmax(1)
    targets = torch.randint(90, (80,), generator=g)
    only = ((dot == dot.max(1, keepdim=True).values).sum(1) == 1) & (targets != top)
    dt, scale = DTYPES[dtype], 2.0 ** power
    got = _run(ps, h.to(dt), table.to(dt), torch.where(only, targets, -100),
               torch.full((80,), 1 / scale), scale)
    fine = got["dh"].isfinite().all(1).cpu()
    assert (got["dh"].cpu()[~fine].isnan().all() and fine[~only].all())
    # what fp32 rounds off lse in base 2 is given back: an exponent of up to 2^-23 of it, which is
    # itself good to 2^-23
    off = UNIT[dt] + 2.0 ** -19 + 2.0 ** -46 * 1.45 * scale * float(dot.max())
    a, b = (table[i].double() * only[:, None].double() for i in (top, targets))
    tol = UNIT[dt] * (a - b).abs() + off * (a.abs() + b.abs()) + 1e-20
    check("dh", got["dh"].cpu()[fine], (a - b)[fine], tol[fine])


@pytest.mark.parametrize("v", [1 + 2.0 ** -7 - 2.0 ** -23, 2 - 2.0 ** -23, 1 + 2.0 ** -8,
                               1 + 2.0 ** -8 + 2.0 ** -16 - 2.0 ** -23, -1.7182817, 1.5])
def test_loss_of_values_that_fill_their_bits(ps, v):  # noqa: F811
    """One product of two fp32 values: the parts left out are at most 2^-24 of it (two products of
    parts of 2^-8 and 2^-17), those kept are added in fp32 with one rounding of the size of the
    sum, cut off at the worst (2^-23), and another below 2^-24."""
    h = torch.tensor([v, 1 + 2.0 ** -7 - 2.0 ** -23, 1.1, 3.3333333, -1.0]).repeat(8)[:, None]
    for w in (v, 1 + 2.0 ** -7 - 2.0 ** -23, 2.0 ** -100 * 1.7182817):
        table = torch.tensor([[w]])
        w = float(table)
        _, lse = ps.linear_cross_entropy_forward(h.cuda(), table.cuda(),
                                                 torch.zeros(40, dtype=torch.int64).cuda())
        val = h[:, 0].double() * w
        check("lse", lse, val, 4 * E * val.abs())


def test_loss_of_the_largest_values(ps):  # noqa: F811
    """No part of a value is past the range that the value is in."""
    top = float(torch.finfo(torch.float32).max)
    h = torch.tensor([top, -top, top * (1 - 2.0 ** -9), 1.0]).repeat(10)[:, None]
    table = torch.tensor([[2.0 ** -120]])
    _, lse = ps.linear_cross_entropy_forward(h.cuda(), table.cuda(),
                                             torch.zeros(40, dtype=torch.int64).cuda())
    val = h[:, 0].double() * 2.0 ** -120
    check("lse", lse, val, 4 * E * val.abs())


@pytest.mark.parametrize("rows, dtype", [((1 << 19) + 1501, "bf16"), ((1 << 19) + 1501, "f16"),
                                         (175101, "f32"), (350001, "f32")])
def test_loss_of_many_rows(ps, rows, dtype):  # noqa: F811
    """More rows than g is kept of at a time."""
    x = _inputs(rows, 50, 8, DTYPES[dtype], 24)
    got = _run(ps, *x)
    c = [t.cuda() for t in x]
    val, tol = cross_entropy(*c[:3], 1.0, c[3])
    for name in val:
        check(name, got[name], val[name].cpu(), tol[name].cpu())
    again = _run(ps, *x, h_grad=False)
    assert torch.equal(got["dtable"], again["dtable"])
    again = _run(ps, *x, table_grad=False)
    assert torch.equal(got["dh"], again["dh"])
