"""Orthogonalised updates on the GPU against the 64-bit iteration, within the bounds that
training_reference.py derives."""
import math

import pytest
import torch

from training_reference import near, orthogonalize, orthogonalize_bound

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FIVE = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def ps():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2608_03199_amd as ps
    ps.load_library()
    return ps


def _matrices(batch, m, n, seed, scale=1e-3):
    """A few strong directions over noise, as momentum has."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    k = min(m, n, 8)
    return scale * ((r(batch, m, k) * torch.exp(-0.4 * torch.arange(k))) @ r(batch, k, n) +
                    0.3 * r(batch, m, n))


SIZES = [(1, 1, 1), (2, 1, 9), (2, 9, 1), (1, 2, 3), (3, 8, 8), (2, 7, 40), (2, 40, 7),
         (1, 63, 65), (2, 65, 63), (1, 128, 128), (2, 129, 127), (1, 127, 300), (1, 300, 127),
         (1, 256, 264), (3, 200, 513), (2, 513, 200), (1, 260, 1000), (1, 1000, 260),
         (40, 33, 32), (1, 640, 640)]


@pytest.mark.parametrize("batch, m, n", SIZES)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_orthogonalize(ps, batch, m, n, dtype):
    g = _matrices(batch, m, n, m + 3 * n).to(DTYPES[dtype])
    val, bound = orthogonalize_bound(g, 5, FIVE, 1e-7)
    got = ps.orthogonalize(g.cuda())
    assert got.shape == g.shape and got.dtype is g.dtype and got.is_contiguous()
    for i in range(batch):
        near(f"matrix {i}", got[i], val[i], bound)
    assert torch.equal(got, ps.orthogonalize(g.cuda()))


@pytest.mark.parametrize("steps, coefficients", [(0, FIVE), (1, FIVE), (2, (1.5, -0.5, 0.0)),
                                                 (12, (1.875, -1.25, 0.375)), (3, (1.0, 0.0, 0.0)),
                                                 (2, (-1.5, 0.5, 0.0))])
@pytest.mark.parametrize("m, n", [(70, 70), (70, 150), (150, 70)])
def test_orthogonalize_steps_and_coefficients(ps, steps, coefficients, m, n):
    g = _matrices(2, m, n, 5)
    val, bound = orthogonalize_bound(g, steps, coefficients, 0.1)
    near("x", ps.orthogonalize(g.cuda(), steps, coefficients, 0.1), val, bound)


def test_orthogonalize_converges(ps):
    """Singular values of 1, the vectors as they were."""
    g = torch.Generator().manual_seed(1)
    u, _ = torch.linalg.qr(torch.randn(60, 60, generator=g, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(90, 60, generator=g, dtype=torch.float64))
    x = u @ torch.diag(torch.logspace(0, -2, 60, dtype=torch.float64)) @ v.T
    got = ps.orthogonalize(x.float().cuda(), 30, (1.875, -1.25, 0.375), 0.0).double().cpu()
    # directions of a hundredth of the strongest: fp32 roundings of the input times 100, and of
    # sums over 60 such directions
    assert float((got - u @ v.T).norm()) < 60 * 100 * 2.0 ** -24 * 8
    s = torch.linalg.svdvals(ps.orthogonalize(x.float().cuda()).double().cpu())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_orthogonalize_strides(ps, dtype):
    base = _matrices(6, 50, 90, 7, 1.0).to(DTYPES[dtype])
    c = base.cuda()
    for view in (lambda t: t, lambda t: t[::2], lambda t: t[:, :, 3:80], lambda t: t[:, 5:40],
                 lambda t: t[1], lambda t: t.mT, lambda t: t.reshape(2, 3, 50, 90),
                 lambda t: t[:1].expand(4, 50, 90), lambda t: t[:, ::3, ::2], lambda t: t[:0],
                 lambda t: t[:, :1], lambda t: t[:, :, :1], lambda t: t[:1, 2:3].expand(1, 7, 90)):
        g = view(base)
        got = ps.orthogonalize(view(c))
        assert got.shape == g.shape
        if g.numel():
            val, bound = orthogonalize_bound(g, 5, FIVE, 1e-7)
            near("x", got, val, bound)


def test_orthogonalize_values_of_any_size(ps):
    """Norms near fp32's ends, zeros, and one matrix that is not a number beside others."""
    g = _matrices(1, 40, 60, 8, 1.0)
    for scale in (1e-30, 1e-12, 1e12, 1e36):
        x = g * scale
        val = orthogonalize(x, 5, FIVE, 0.0)
        single = orthogonalize(g, 5, FIVE, 0.0, torch.float32).double()
        exact = orthogonalize(g, 5, FIVE, 0.0)
        bound = 4 * float((single - exact).norm() / exact.norm()) + 8 * 2.0 ** -24
        near(str(scale), ps.orthogonalize(x.cuda(), eps=0.0), val, bound)
    zero = torch.zeros(2, 30, 20)
    assert not ps.orthogonalize(zero.cuda()).any()
    x = _matrices(3, 40, 60, 9, 1.0)
    want = ps.orthogonalize(x.cuda())
    for bad in (math.nan, math.inf):
        y = x.clone()
        y[1, 3, 5] = bad
        got = ps.orthogonalize(y.cuda())
        assert not got[1].isfinite().any()
        assert torch.equal(got[[0, 2]], want[[0, 2]])


def test_orthogonalize_many_matrices(ps):
    """A stack that is taken in turns gives what its matrices give one by one."""
    g = _matrices(3000, 8, 8, 10)
    got = ps.orthogonalize(g.cuda())
    for i in (0, 1, 1499, 2999):
        assert torch.equal(got[i], ps.orthogonalize(g[i].cuda()))
    big = _matrices(1, 8, 8, 11).expand(70000, 8, 8).cuda()  # more than one launch takes
    got = ps.orthogonalize(big)
    assert torch.equal(got, got[:1].expand(70000, 8, 8))


def test_orthogonalize_streams_and_graph(ps):
    g = _matrices(2, 150, 100, 12).cuda()
    want = ps.orthogonalize(g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ps.orthogonalize(g, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ps.orthogonalize(g)
    for k in range(4):
        g.copy_(_matrices(2, 150, 100, 20 + k))
        want = ps.orthogonalize(g).clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want), k


def test_orthogonalize_refusals(ps):
    g = torch.ones(4, 5).cuda()
    for bad in (g.cpu(), g[0], g[:0], g[:, :0]):
        with pytest.raises(ValueError):
            ps.orthogonalize(bad)
    with pytest.raises(TypeError):
        ps.orthogonalize(g.double())
    with pytest.raises(ValueError):
        ps.orthogonalize(g, 5, (1.0, 2.0))
    for bad in (dict(steps=-1), dict(steps=1001), dict(eps=-1.0), dict(eps=math.nan),
                dict(coefficients=(math.nan, 0.0, 0.0)), dict(coefficients=(5.0, 0.0, 0.0)),
                dict(coefficients=(20.0, -30.0, 10.5)), dict(steps=9, coefficients=(1.2, 0.0, 0.0))):
        with pytest.raises(ps.SieveError):
            ps.orthogonalize(g, **bad)
