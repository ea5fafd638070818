"""The table's lookup and its gradient on the GPU against the 64-bit oracle, value by value within
the bounds that training_reference.py derives."""
import math

import pytest
import torch

from encoder_reference import check
from training_reference import embed

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
PAIRS = [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "f16"), ("f32", "bf16")]


@pytest.fixture(scope="module")
def ps():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2608_03199_amd as ps
    ps.load_library()
    return ps


def _rnd(seed):
    g = torch.Generator().manual_seed(seed)
    return g, lambda *s: torch.randn(*s, generator=g)


def _ids(kind, count, vocab, g):
    if kind == "uniform":
        return torch.randint(vocab, (count,), generator=g)
    if kind == "frequent":  # half of them one number, a tenth another
        ids = torch.randint(vocab, (count,), generator=g)
        u = torch.rand(count, generator=g)
        return torch.where(u < 0.5, vocab // 3, torch.where(u < 0.6, vocab - 1, ids))
    if kind == "one":
        return torch.full((count,), vocab - 1)
    if kind == "none":
        return torch.where(torch.rand(count, generator=g) < 0.5, -1, vocab)
    assert kind == "padded"
    ids = torch.randint(vocab, (count,), generator=g)
    u = torch.rand(count, generator=g)
    return torch.where(u < 0.3, -1, torch.where(u < 0.35, vocab, ids))


CASES = [(1, 1, 1, "uniform"), (1, 50, 64, "uniform"), (24, 32768, 768, "uniform"),
         (31, 7, 7, "uniform"), (32, 3, 8, "one"), (33, 3, 515, "one"), (64, 40, 16, "padded"),
         (2047, 1023, 24, "padded"), (2048, 1024, 64, "frequent"), (2049, 1025, 40, "uniform"),
         (5000, 2000, 515, "frequent"), (1023, 5, 2048, "one"), (1024, 5, 2056, "one"),
         (3000, 9, 1001, "none"), (70001, 50000, 64, "frequent"), (70001, 2, 33, "padded"),
         (40000, 1100000, 8, "frequent"), (300000, 40000, 12, "frequent"),
         (5000, 1 << 20, 4, "padded"), (100, 70000, 1000, "uniform")]


@pytest.mark.parametrize("count, vocab, n, kind", CASES)
@pytest.mark.parametrize("tdtype, dtype", PAIRS)
def test_embed(ps, count, vocab, n, kind, tdtype, dtype):
    g, rnd = _rnd(count + 3 * n)
    td, dt = DTYPES[tdtype], DTYPES[dtype]
    table, dy = rnd(vocab, n).to(td), rnd(count, n).to(dt)
    ids = _ids(kind, count, vocab, g)
    scale = math.sqrt(n)
    val, tol = embed(ids, table, scale, dt, dy)
    for it in (torch.int64, torch.int32):
        i = ids.to(it).cuda()
        check("out", ps.embed_forward(i, table.cuda(), scale, dtype=dt), val["out"], tol["out"])
        got = ps.embed_backward(dy.cuda(), i, vocab, scale, dtype=td)
        check("dtable", got, val["dtable"], tol["dtable"])
        assert torch.equal(got, ps.embed_backward(dy.cuda(), i, vocab, scale, dtype=td))
    # added to a gradient that is there: only the rows that a number names are touched
    into = rnd(vocab, n).to(td)
    _, tol_sum = embed(ids, table, scale, dt, dy, into)
    held = into.cuda()
    got = ps.embed_backward(dy.cuda(), ids.cuda(), vocab, scale, into=held)
    assert got.data_ptr() == held.data_ptr()
    check("into", got, val["dtable"] + into.double(), tol_sum["dtable"])
    idle = torch.ones(vocab, dtype=torch.bool)
    idle[ids[(ids >= 0) & (ids < vocab)]] = False
    assert torch.equal(got.cpu()[idle], into[idle])


def test_embed_numbers_far_outside(ps):
    """Numbers that no 32-bit table row has, the lowest and highest of their type among them."""
    g, rnd = _rnd(1)
    table, dy = rnd(10, 16), rnd(8, 16)
    ids = torch.tensor([3, 1 << 40, -(1 << 40), (1 << 32) + 3, 2 ** 63 - 1, -2 ** 63, 9, 10])
    out = ps.embed_forward(ids.cuda(), table.cuda())
    want = torch.zeros(8, 16)
    want[0], want[6] = table[3], table[9]
    assert torch.equal(out.cpu(), want)
    got = ps.embed_backward(dy.cuda(), ids.cuda(), 10)
    want = torch.zeros(10, 16)
    want[3], want[9] = dy[0], dy[6]
    assert torch.equal(got.cpu(), want)
    ids = torch.tensor([3, 2 ** 31 - 1, -2 ** 31, 9], dtype=torch.int32)
    assert torch.equal(ps.embed_forward(ids.cuda(), table.cuda()).cpu()[[0, 3]], table[[3, 9]])


def test_embed_left_out_rows_are_not_used(ps):
    """What dy holds for tokens outside of the table reaches nothing, nor does a row that no
    number names."""
    table = torch.ones(100, 24)
    table[50] = math.nan
    dy = torch.ones(200, 24)
    ids = torch.arange(200) % 50
    ids[::3] = -1
    dy[::3] = math.inf
    dy[3] = math.nan
    out = ps.embed_forward(ids.cuda(), table.cuda())
    assert torch.equal(out[:, 0].cpu(), (ids >= 0).float())
    got = ps.embed_backward(dy.cuda(), ids.cuda(), 100).cpu()
    assert torch.equal(got[:, 0], torch.bincount(ids[ids >= 0], minlength=100).float())
    # one that counts stays in its row
    ids[3] = 7
    got = ps.embed_backward(dy.cuda(), ids.cuda(), 100).cpu()
    assert got[7].isnan().all() and got[:7].isfinite().all() and got[8:].isfinite().all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_embed_strides_and_shapes(ps, dtype):
    dt = DTYPES[dtype]
    g, rnd = _rnd(3)
    wide, dwide = rnd(30, 200).to(dt), rnd(4, 5, 3, 200).to(dt)
    ids = torch.randint(-1, 30, (4, 5, 3), generator=g)
    for lo, hi in ((0, 64), (8, 72), (3, 67), (1, 200)):
        table, dy = wide[:, lo:hi], dwide[..., lo:hi]
        val, tol = embed(ids, table, 2.0, dt, dy)
        cw, cd = wide.cuda()[:, lo:hi], dwide.cuda()[..., lo:hi]
        out = ps.embed_forward(ids.cuda(), cw, 2.0)
        assert out.shape == (4, 5, 3, hi - lo)
        check("out", out, val["out"], tol["out"])
        check("dtable", ps.embed_backward(cd, ids.cuda(), 30, 2.0), val["dtable"], tol["dtable"])
    # transposed tables and numbers, expanded gradients
    val, tol = embed(ids.transpose(0, 2), wide[:, :30].t(), 1.0, dt)
    check("out", ps.embed_forward(ids.cuda().transpose(0, 2), wide.cuda()[:, :30].t()),
          val["out"], tol["out"])
    one = rnd(1, 1, 1, 64).to(dt).expand(4, 5, 3, 64)
    val, tol = embed(ids, wide[:, :64], 1.0, dt, one)
    check("dtable", ps.embed_backward(one.cuda(), ids.cuda(), 30), val["dtable"], tol["dtable"])


def test_embed_nothing(ps):
    table, none = torch.ones(5, 8).cuda(), torch.zeros(0, dtype=torch.int64).cuda()
    assert ps.embed_forward(none, table).shape == (0, 8)
    got = ps.embed_backward(torch.zeros(0, 8).cuda(), none, 5)
    assert got.shape == (5, 8) and not got.any()
    assert torch.equal(ps.embed_backward(torch.zeros(0, 8).cuda(), none, 5, into=table),
                       torch.ones(5, 8).cuda())
    assert ps.embed_forward(torch.tensor(2).cuda(), table).shape == (8,)


def test_embed_autograd_streams_and_graph(ps):
    g, rnd = _rnd(5)
    table, dy = rnd(300, 96), rnd(700, 96).bfloat16()
    ids = torch.randint(-1, 300, (700,), generator=g)
    val, tol = embed(ids, table, 3.0, torch.bfloat16, dy)
    t = table.cuda().requires_grad_()
    out = ps.embed(ids.cuda(), t, 3.0, torch.bfloat16)
    out.backward(dy.cuda())
    check("out", out, val["out"], tol["out"])
    assert t.grad.dtype is torch.float32
    check("dtable", t.grad, val["dtable"], tol["dtable"])
    # another stream than the current one
    s = torch.cuda.Stream()
    i, d, w = ids.cuda(), dy.cuda(), table.cuda()
    s.wait_stream(torch.cuda.current_stream())
    got = ps.embed_backward(d, i, 300, 3.0, dtype=torch.float32, stream=s)
    s.synchronize()
    check("dtable", got, val["dtable"], tol["dtable"])

    def step():
        return (ps.embed_forward(i, w, 3.0, torch.bfloat16),
                ps.embed_backward(d, i, 300, 3.0, dtype=torch.float32))

    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(4):
        i.copy_(torch.randint(-1, 300, (700,), generator=g))
        d.copy_(rnd(700, 96).bfloat16())
        want = [x.clone() for x in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), k


def test_embed_against_differences(ps):
    """The lookup is linear in the table: its change along a direction is the gradient's."""
    g, rnd = _rnd(6)
    table, way, dy = rnd(40, 12), rnd(40, 12), rnd(90, 12)
    ids = torch.randint(-1, 40, (90,), generator=g).cuda()

    def at(s):
        out = ps.embed_forward(ids, (table + s * way).cuda(), 1.5)
        return float((out.double().cpu() * dy.double()).sum())

    grad = ps.embed_backward(dy.cuda(), ids, 40, 1.5).double().cpu()
    slope = float((grad * way.double()).sum())
    # values of at most about 8 rounded three times in fp32, 1,080 of them, over a step of 2
    bound = 90 * 12 * 8 * 1.5 * 4 * 4 * 2.0 ** -24
    assert abs((at(1.0) - at(-1.0)) / 2 - slope) < bound


def test_embed_refusals(ps):
    table, ids = torch.zeros(5, 8).cuda(), torch.zeros(3, dtype=torch.int64).cuda()
    dy = torch.zeros(3, 8).cuda()
    for bad in ((ids.float(), table), (ids.to(torch.int16), table), (ids, table.double()),
                (ids, table.half(), 1.0, torch.float32), (ids, table, 1.0, torch.float64)):
        with pytest.raises(TypeError):
            ps.embed_forward(*bad)
    for bad in ((ids, table[0]), (ids.cpu(), table), (ids, table.cpu()), (ids, table[:, :0]),
                (ids, table[:0])):
        with pytest.raises(ValueError):
            ps.embed_forward(*bad)
    with pytest.raises(ps.SieveError):
        ps.embed_forward(ids, torch.zeros(1, 65537).cuda())
    for bad in (dict(vocab=0), dict(ids=ids[:2]), dict(dy=dy.cpu()), dict(ids=ids.cpu()),
                dict(into=table[:4]), dict(into=table.half(), dtype=torch.float32),
                dict(into=torch.zeros(8, 5).cuda().t())):
        with pytest.raises(ValueError):
            ps.embed_backward(**{**dict(dy=dy, ids=ids, vocab=5), **bad})
    for bad in (dict(dy=dy.double()), dict(dtype=torch.float16), dict(ids=ids.bool())):
        with pytest.raises(TypeError):
            ps.embed_backward(**{**dict(dy=dy, ids=ids, vocab=5), **bad})
