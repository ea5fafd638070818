"""The text-encoder operators where their arithmetic is easiest to get wrong: statistics of 16-bit
rows, values that are not numbers, and biases far below the scores."""
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
