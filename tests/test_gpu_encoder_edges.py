"""The text-encoder operators where their arithmetic is easiest to get wrong: statistics of 16-bit
rows, values that are not numbers, and biases far below the scores."""
import math

import pytest
import torch

from encoder_reference import UNIT, attention, check

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ps():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2608_03199_amd as ps
    ps.load_library()
    return ps


def _rnd(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g)


def _offsets(lens):
    return torch.tensor([0] + list(lens)).cumsum(0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("qlens, klens, heads, kv_heads, d, causal, buckets", [
    ([200, 8, 1], [200, 8, 1], 2, 2, 64, False, 0),       # whole rows
    ([130, 40], [130, 40], 4, 1, 128, True, 16),
    ([1, 2, 3], [700, 90, 5], 4, 2, 64, False, 0),        # waves that share the keys of few rows
    ([1], [5000], 8, 2, 128, False, 0),                   # and items that do
    ([2300], [2300], 2, 1, 64, True, 0)])
def test_attention_lse_in_16_bits_is_of_unrounded_probabilities(ps, dtype, qlens, klens, heads,
                                                                kv_heads, d, causal, buckets):
    """lse is a statistic in fp32: the oracle's bound for it without its term for probabilities
    that were rounded to 16 bits first."""
    dt, rnd = DTYPES[dtype], _rnd(31)
    qo, ko = _offsets(qlens), _offsets(klens)
    q = rnd(int(qo[-1]), heads, d).to(dt)
    k, v = rnd(int(ko[-1]), kv_heads, d).to(dt), rnd(int(ko[-1]), kv_heads, d).to(dt)
    bias = rnd(buckets, heads).to(dt) if buckets else None
    plan = ps.AttentionPlan(qo, ko, heads=heads, kv_heads=kv_heads, head_dim=d, dtype=dt,
                            causal=causal, num_buckets=buckets, max_distance=40 if buckets else 0)
    _, lse = plan.forward(q.cuda(), k.cuda(), v.cuda(), bias=None if bias is None else bias.cuda())
    val, tol = attention(q, k, v, qo, ko, causal, None, None, bias, 40)
    check("lse", lse, val["lse"], tol["lse"] - (tol["lse"] > 0) * UNIT[dt])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("lens, heads, kv_heads, d", [
    ([150, 20, 400], 2, 2, 64), ([150, 20, 400], 4, 1, 128), ([150, 20, 400], 3, 1, 20),
    ([2300], 2, 1, 96)])
@pytest.mark.parametrize("buckets", [0, 8])
def test_attention_causal_earlier_rows_do_not_reach_later_keys(ps, dtype, lens, heads, kv_heads, d,
                                                               buckets):
    """A row whose q and dout are not numbers gives nothing to the keys after its position: their
    gradients are as without it."""
    dt, rnd = DTYPES[dtype], _rnd(32)
    o = _offsets(lens)
    n = int(o[-1])
    q, k, v = rnd(n, heads, d).to(dt), rnd(n, kv_heads, d).to(dt), rnd(n, kv_heads, d).to(dt)
    dout = rnd(n, heads, d).to(dt)
    bias = rnd(buckets, heads).to(dt) if buckets else None
    odd_q, odd_dout = q.clone(), dout.clone()
    later = torch.zeros(n, dtype=torch.bool)
    for s, length in enumerate(lens):
        row = int(o[s]) + length // 4 + 2
        odd_q[row, 0], odd_dout[row, 0] = math.nan, math.inf
        q[row, 0], dout[row, 0] = 0, 0  # what the oracle has there does not matter after it
        later[row + 1:int(o[s + 1])] = True
    plan = ps.AttentionPlan(o, heads=heads, kv_heads=kv_heads, head_dim=d, dtype=dt, causal=True,
                            num_buckets=buckets, max_distance=30 if buckets else 0)
    b = None if bias is None else bias.cuda()
    out, lse = plan.forward(odd_q.cuda(), k.cuda(), v.cuda(), bias=b)
    _, dk, dv, _ = plan.backward(odd_dout.cuda(), odd_q.cuda(), k.cuda(), v.cuda(), out, lse,
                                 bias=b)
    val, tol = attention(q, k, v, o, o, True, bias=bias, distance=30, dout=dout)
    check("dk", dk.cpu()[later], val["dk"][later], tol["dk"][later])
    check("dv", dv.cpu()[later], val["dv"][later], tol["dv"][later])
    # and what sees it shows it
    assert not torch.isfinite(dk.cpu()[int(o[0]) + lens[0] // 4 + 2, 0]).all()
    assert not torch.isfinite(dv.cpu()[int(o[0]) + lens[0] // 4 + 2, 0]).any()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("value", ["lowest", -1e30, -1e9, -3e6, 1e9, "largest"])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_bias_far_from_the_scores(ps, dtype, value, causal):
    """A row all of whose keys have a bias of the type's lowest value, or one that fp32 cannot add
    scores to: as with the limit that the bias is held to, in both passes."""
    dt, rnd = DTYPES[dtype], _rnd(33)
    info = torch.finfo(dt)
    value = info.min if value == "lowest" else info.max if value == "largest" else value
    value = max(info.min, min(info.max, value))
    o = _offsets([60, 200])
    q, k, v = rnd(260, 2, 32).to(dt), rnd(260, 2, 32).to(dt), rnd(260, 2, 32).to(dt)
    dout = rnd(260, 2, 32).to(dt)
    bias = rnd(8, 2).to(dt)
    bias[:, 1] = value  # every key of head 1
    held = bias.double().clamp(-2.0 ** 20, 2.0 ** 20)
    plan = ps.AttentionPlan(o, heads=2, head_dim=32, dtype=dt, causal=causal, num_buckets=8,
                            max_distance=30)
    out, lse = plan.forward(q.cuda(), k.cuda(), v.cuda(), bias=bias.cuda())
    grads = plan.backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse, bias=bias.cuda())
    val, tol = attention(q, k, v, o, o, causal, bias=held, distance=30, dout=dout)
    for name, got in zip(("out", "dq", "dk", "dv", "dbias", "lse"), (out, *grads, lse)):
        check(name, got, val[name], tol[name])
    # head 0 is none of it
    val, tol = attention(q[:, :1], k[:, :1], v[:, :1], o, o, causal, bias=bias[:, :1], distance=30,
                         dout=dout[:, :1])
    for name, got in zip(("out", "dq", "dk", "dv"), (out,) + tuple(grads[:3])):
        check(name, got[:, :1], val[name], tol[name])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("buckets, distance", [(8, 30), (128, 40)])
def test_attention_bias_that_is_not_a_number(ps, dtype, buckets, distance):
    """The limit of a bias leaves NaN, and -infinity forbids as before; the lowest value does
    not."""
    dt, rnd = DTYPES[dtype], _rnd(34)
    q = rnd(50, 4, 32).to(dt).cuda()
    bias = rnd(buckets, 4).to(dt)
    bias[:, 1], bias[:, 2], bias[:, 3] = math.nan, -math.inf, torch.finfo(dt).min
    plan = ps.AttentionPlan([0, 50], heads=4, head_dim=32, dtype=dt, num_buckets=buckets,
                            max_distance=distance)
    out, lse = plan.forward(q, q, q, bias=bias.cuda())
    assert torch.isfinite(out[:, 0]).all() and torch.isnan(out[:, 1]).all()
    assert not out[:, 2].any() and torch.isneginf(lse[:, 2]).all()
    assert torch.isfinite(out[:, 3]).all() and out[:, 3].any(1).all()
    assert (lse[:, 3] + 2.0 ** 20).abs().max() < 64


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("d", [64, 128, 40])
def test_attention_few_causal_rows_before_odd_values(ps, dtype, d):
    """The last queries of documents whose last key is not a number: those before it are as
    without it, where waves share the keys of a tile and where work-groups do."""
    dt, rnd = DTYPES[dtype], _rnd(35)
    qo, ko = _offsets([3, 2, 5]), _offsets([300, 5000, 66])
    q, dout = rnd(10, 4, d).to(dt), rnd(10, 4, d).to(dt)
    k, v = rnd(5366, 2, d).to(dt), rnd(5366, 2, d).to(dt)
    val, tol = attention(q, k, v, qo, ko, True, dout=dout)
    odd_k, odd_v = k.clone(), v.clone()
    last = ko[1:] - 1
    odd_k[last], odd_v[last] = math.nan, math.inf
    plan = ps.AttentionPlan(qo, ko, heads=4, kv_heads=2, head_dim=d, dtype=dt, causal=True)
    out, lse = plan.forward(q.cuda(), odd_k.cuda(), odd_v.cuda())
    dq = plan.backward(dout.cuda(), q.cuda(), odd_k.cuda(), odd_v.cuda(), out, lse)[0]
    before = torch.ones(10, dtype=torch.bool)
    before[qo[1:] - 1] = False
    for name, got in (("out", out), ("lse", lse), ("dq", dq)):
        check(name, got.cpu()[before], val[name][before], tol[name][before])
    assert not torch.isfinite(out.cpu()[~before]).any()


def test_attention_gradient_probabilities_keep_32_bits(ps):
    """The backward pass's probabilities in fp32, seen through dv: scores of 0 over n keys, an
    output's gradient of 1, so that dv is the probability 1 / n.

    What they are made of: lse in units of log2 (below 4), its product with ln 2 and back, each
    rounded to nearest, half a unit of which is at most 2 E (E = 2^-24), a quarter on average, the
    exponential and the result.  On average that is at most 3 E ln 2 + E, below 3.1 E.  A
    statistic moved by a constant that makes it larger (by 24: 16 E, 5.5 E on average) is not."""
    lens = [n for n in range(3, 16) if n & (n - 1)]
    plan = ps.AttentionPlan(torch.arange(len(lens) + 1), _offsets(lens), heads=1, head_dim=4,
                            dtype=torch.float32)
    q, k = torch.zeros(len(lens), 1, 4).cuda(), torch.zeros(sum(lens), 1, 4).cuda()
    v = torch.randn(sum(lens), 1, 4, generator=torch.Generator().manual_seed(36)).cuda()
    out, lse = plan.forward(q, k, v)
    dv = plan.backward(torch.ones_like(q), q, k, v, out, lse)[2]
    n = torch.tensor([float(n) for n in lens for _ in range(n)], dtype=torch.float64)
    off = (dv.double().cpu()[:, 0] * n[:, None] - 1).abs().amax(1)
    per = torch.stack([x.max() for x in off.split(lens)])
    assert float(per.mean()) < 3.1 * 2.0 ** -24


@pytest.mark.parametrize("causal", [False, True])
def test_attention_small_half_precision_gradients_beside_an_infinite_one(ps, causal):
    """binary16 scales dS by the largest of a sequence: a row whose dS is infinite is not it, so
    that gradients of 1e-6 keep their relative precision where that row does not reach."""
    rnd = _rnd(37)
    o = _offsets([300, 40])
    q, k, v = rnd(340, 2, 64).half(), rnd(340, 2, 64).half(), rnd(340, 2, 64).half()
    dout = (rnd(340, 2, 64) * 1e-6).half()
    dout[10, 0] = 0  # what the oracle has there does not matter past its reach
    odd = dout.clone()
    odd[10, 0, 0] = math.inf  # dP of that row is infinite of both signs, dS infinite or NaN
    val, tol = attention(q, k, v, o, o, causal, dout=dout)
    plan = ps.AttentionPlan(o, heads=2, head_dim=64, dtype=torch.float16, causal=causal)
    out, lse = plan.forward(q.cuda(), k.cuda(), v.cuda())
    dq, dk, dv, _ = plan.backward(odd.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse)
    rows = torch.ones(340, dtype=torch.bool)
    rows[10] = False
    check("dq", dq.cpu()[rows], val["dq"][rows], tol["dq"][rows])
    check("dq", dq.cpu()[:, 1], val["dq"][:, 1], tol["dq"][:, 1])
    keys = torch.ones(340, dtype=torch.bool)
    keys[:300 if not causal else 11] = False
    for name, got in (("dk", dk), ("dv", dv)):
        check(name, got.cpu()[keys], val[name][keys], tol[name][keys])
        check(name, got.cpu()[:, 1], val[name][:, 1], tol[name][:, 1])
