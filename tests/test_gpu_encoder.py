"""The text-encoder operators on the GPU against the 64-bit oracle, value by value within the
bounds that encoder_reference.py derives."""
import math

import pytest
import torch

from encoder_reference import attention, bucket, check, norm

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


# ---- layer norm ----------------------------------------------------------------------------

ROWS_N = [(1, 1), (1, 768), (3, 7), (5, 64), (24, 768), (70, 515), (33, 512), (9, 1024), (130, 96),
          (6, 2048), (5, 2056), (7, 4096), (3, 4099), (4, 8192), (3, 9001), (2, 20000),
          (4200, 128)]


@pytest.mark.parametrize("rows, n", ROWS_N)
@pytest.mark.parametrize("dtype, wdtype", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"),
                                           ("bf16", "bf16"), ("bf16", "f32")])
def test_norm(ps, rows, n, dtype, wdtype):
    rnd = _rnd(rows * 7 + n)
    dt, wt = DTYPES[dtype], DTYPES[wdtype]
    x, r = (rnd(rows, n) * 1.5 + 0.3).to(dt), rnd(rows, n).to(dt)
    w, b = (rnd(n) * 0.3 + 1).to(wt), (rnd(n) * 0.2).to(wt)
    dy, dh = rnd(rows, n).to(dt), rnd(rows, n).to(dt)
    c = lambda t: t.cuda()  # noqa: E731
    for residual in (None, r):
        y, h, mean, rstd = ps.layer_norm_forward(c(x), c(w), c(b), 1e-5,
                                                 None if residual is None else c(residual))
        skip = None if residual is None else dh
        dx, dw, db = ps.layer_norm_backward(c(dy), h, c(w), mean, rstd,
                                            None if skip is None else c(skip))
        val, tol = norm(x, w, b, 1e-5, residual, dy, skip)
        assert torch.equal(h.double().cpu().reshape(rows, n), val["h"])
        for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dweight", dw),
                          ("dbias", db)):
            check(name, got, val[name], tol[name])


def test_norm_without_bias_and_parts_of_the_gradient(ps):
    rnd = _rnd(2)
    x, w, dy = rnd(40, 96).half(), rnd(96).half(), rnd(40, 96).half()
    y, h, mean, rstd = ps.layer_norm_forward(x.cuda(), w.cuda())
    val, tol = norm(x, w, None, 1e-5, None, dy)
    check("y", y, val["y"], tol["y"])
    for want_w, want_b in ((True, False), (False, True), (False, False)):
        dx, dw, db = ps.layer_norm_backward(dy.cuda(), h, w.cuda(), mean, rstd,
                                            weight_grad=want_w, bias_grad=want_b)
        check("dx", dx, val["dx"], tol["dx"])
        assert (dw is not None) == want_w and (db is not None) == want_b
        if want_w:
            check("dweight", dw, val["dweight"], tol["dweight"])
        if want_b:
            check("dbias", db, val["dbias"], tol["dbias"])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_norm_strides_and_shapes(ps, dtype):
    """Rows that are slices, expanded rows, more than two axes, unaligned starts."""
    dt, rnd = DTYPES[dtype], _rnd(4)
    wide = rnd(12, 3, 200).to(dt)
    w, b = (rnd(64) + 1).to(dt), rnd(64).to(dt)
    for name, t in (("slice", wide[:, 1, 8:72]), ("odd start", wide[:, 1, 3:67]),
                    ("three axes", wide[:, :, 16:80]), ("expanded", wide[:1, 0, :64].expand(9, 64)),
                    ("across", wide[:, 0, :].t()[:64].t()), ("columns", rnd(64, 5).to(dt).t())):
        y, h, mean, rstd = ps.layer_norm_forward(t.cuda() if name == "columns" else
                                                 _like_on_gpu(t), w.cuda(), b.cuda())
        val, tol = norm(t.contiguous(), w, b, 1e-5, None, t.contiguous())
        check(name, y, val["y"], tol["y"])
        dx, dw, db = ps.layer_norm_backward(_like_on_gpu(t), h, w.cuda(), mean, rstd)
        check(name, dx, val["dx"], tol["dx"])
        check(name, dw, val["dweight"], tol["dweight"])


def _like_on_gpu(t):
    """The same view of the same storage, on the GPU."""
    base = torch.empty(0, dtype=t.dtype).set_(t.untyped_storage()).cuda()
    return base.as_strided(t.shape, t.stride(), t.storage_offset())


def test_norm_no_rows(ps):
    w = torch.ones(16).cuda()
    x = torch.empty(0, 16).cuda()
    y, h, mean, rstd = ps.layer_norm_forward(x, w, w)
    assert y.shape == (0, 16) and mean.shape == (0,)
    dx, dw, db = ps.layer_norm_backward(x, h, w, mean, rstd)
    assert dx.shape == (0, 16) and not dw.any() and not db.any()
    w = torch.ones(9000).cuda()
    x = torch.empty(0, 9000).cuda()
    y, h, mean, rstd = ps.layer_norm_forward(x, w, w)
    dx, dw, db = ps.layer_norm_backward(x, h, w, mean, rstd)
    assert not dw.any() and not db.any()


def test_norm_odd_values_stay_in_their_rows(ps):
    x = torch.randn(6, 64, generator=torch.Generator().manual_seed(1))
    x[1, 5], x[3, 0], x[4] = math.nan, math.inf, 2.5
    w = torch.ones(64)
    y, _, mean, rstd = ps.layer_norm_forward(x.cuda(), w.cuda(), w.cuda())
    y = y.cpu()
    assert torch.isnan(y[1]).all() and not torch.isfinite(y[3]).any()
    assert torch.isfinite(y[[0, 2, 4, 5]]).all()
    assert torch.equal(y[4], torch.ones(64))  # a row of equal values: its bias


def test_norm_autograd(ps):
    rnd = _rnd(5)
    x, r = rnd(3, 5, 48).double(), rnd(3, 5, 48).double()
    w, b = rnd(48).double(), rnd(48).double()
    t = [v.float().cuda().requires_grad_() for v in (x, r, w, b)]
    y, h = ps.layer_norm(t[0], t[2], t[3], residual=t[1])
    (y * 2 + h.square()).sum().backward()
    u = [v.clone().requires_grad_() for v in (x, r, w, b)]
    z = u[0] + u[1]
    (torch.nn.functional.layer_norm(z, (48,), u[2], u[3]) * 2 + z.square()).sum().backward()
    for got, want in zip(t, u):
        assert torch.allclose(got.grad.double().cpu(), want.grad, rtol=1e-4, atol=1e-4)


def test_norm_refusals(ps):
    x, w = torch.zeros(4, 8).cuda(), torch.ones(8).cuda()
    for bad in (dict(x=x.cpu()), dict(weight=w[:4]), dict(weight=w.half()), dict(bias=w[:7]),
                dict(residual=x[:3]), dict(residual=x.half()), dict(x=x.double()),
                dict(x=x.half(), weight=w, bias=w.half())):
        args = dict(x=x, weight=w, bias=w)
        args.update(bad)
        with pytest.raises((ValueError, TypeError)):
            ps.layer_norm_forward(**args)
    with pytest.raises(ps.SieveError):
        ps.layer_norm_forward(torch.zeros(1, 70000).cuda(), torch.ones(70000).cuda())
    y, h, mean, rstd = ps.layer_norm_forward(x, w, w)
    for bad in (dict(dy=x[:2]), dict(mean=mean[:2]), dict(rstd=rstd.double()), dict(dh=x.half())):
        args = dict(dy=x, h=h, weight=w, mean=mean, rstd=rstd)
        args.update(bad)
        with pytest.raises((ValueError, TypeError)):
            ps.layer_norm_backward(**args)


# ---- attention -------------------------------------------------------------------------------


def _offsets(lens):
    return torch.tensor([0] + list(lens)).cumsum(0)


def _run(ps, dtype, qlens, klens, heads, kv_heads, d, seed=0, causal=False, buckets=0, distance=0,
         masked=None, train=True, scale=None, fused=False, odd=False, table=None, spread=1.2):
    dt, rnd = DTYPES[dtype], _rnd(seed)
    qo, ko = _offsets(qlens), _offsets(klens)
    rows, keys = int(qo[-1]), int(ko[-1])
    if fused:
        qkv = rnd(keys, 3, heads, d).to(dt)
        q, k, v = qkv[:, 0], qkv[:, 1], qkv[:, 2]
    else:
        q = (rnd(rows, heads, d) * spread).to(dt)
        k, v = (rnd(keys, kv_heads, d) * spread).to(dt), rnd(keys, kv_heads, d).to(dt)
    dout = rnd(rows, heads, d).to(dt)
    bias = (rnd(buckets, heads) * 0.7).to(dt) if buckets else None
    if table is not None:
        bias = table(bias)
    mask = None
    if masked is not None:
        mask = masked(keys, ko)
        k, v = k.clone(), v.clone()
        k[~mask], v[~mask] = math.nan, -math.inf
    plan = ps.AttentionPlan(qo, ko, heads=heads, kv_heads=kv_heads, head_dim=d, dtype=dt,
                            causal=causal, scale=scale, num_buckets=buckets, max_distance=distance)
    on = (lambda t: None if t is None else _like_on_gpu(t) if fused and t.dim() == 3 else t.cuda())
    out, lse = plan.forward(on(q), on(k), on(v), key_mask=on(mask), bias=on(bias))
    got = {"out": out, "lse": lse}
    if train:
        got["dq"], got["dk"], got["dv"], got["dbias"] = plan.backward(
            dout.cuda(), on(q), on(k), on(v), out, lse, key_mask=on(mask), bias=on(bias))
        again = plan.backward(dout.cuda(), on(q), on(k), on(v), out, lse, key_mask=on(mask),
                              bias=on(bias))
        for a, b in zip(again, (got["dq"], got["dk"], got["dv"], got["dbias"])):
            assert (a is None and b is None) or torch.equal(a, b)
    torch.cuda.synchronize()
    if odd:
        return got, (q, k, v, qo, ko, dout, bias, mask)
    val, tol = attention(q, k, v, qo, ko, causal, scale, mask, bias, distance,
                         dout if train else None)
    for name, t in got.items():
        if t is not None:
            check(name, t, val[name], tol[name])
    return got, None


def _some(keys, offsets):
    m = torch.rand(keys, generator=torch.Generator().manual_seed(9)) > 0.3
    for s in range(1, len(offsets) - 1, 3):
        m[offsets[s]:offsets[s + 1]] = False  # whole sequences
    return m


LENS = [1, 31, 0, 64, 130, 5, 97]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads, kv_heads", [(2, 2), (4, 1), (6, 2), (5, 1)])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("buckets", [0, 16])
def test_attention(ps, dtype, heads, kv_heads, d, causal, buckets):
    _run(ps, dtype, LENS, LENS, heads, kv_heads, d, 1, causal, buckets, 40 if buckets else 0,
         _some if buckets == 0 or d == 32 else None)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("d", [1, 3, 8, 20, 33, 40, 72, 80, 96, 100, 127])
def test_attention_head_sizes(ps, dtype, d):
    _run(ps, dtype, [50, 3, 70], [50, 3, 70], 2, 1, d, d, causal=d % 2 == 0, buckets=8, distance=30)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("qlens, klens", [
    ([1, 1, 1], [1, 500, 77]),          # one query a sequence, split keys
    ([2, 5, 1], [900, 0, 3]),           # no keys at all
    ([70, 9, 40], [20, 9, 0]),          # more queries than keys: causal rows that see none
    ([0, 4, 0], [30, 7, 200]),          # keys that no query sees
    ([300], [2000]), ([1], [1]), ([], [])])
def test_attention_lengths(ps, dtype, causal, qlens, klens):
    _run(ps, dtype, qlens, klens, 4, 2, 64, 3, causal, 16, 40)
    _run(ps, dtype, qlens, klens, 3, 3, 32, 4, causal)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_long(ps, dtype, d):
    """Key ranges and row ranges that are shared out and joined, forward and backward."""
    _run(ps, dtype, [2300], [2300], 2, 1, d, 5, True)
    _run(ps, dtype, [1500, 40], [1500, 40], 2, 2, d, 6, False, 32, 128, _some)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_attention_few_rows_over_many_keys(ps, dtype):
    _run(ps, dtype, [1, 2, 1, 3], [5000, 1, 3001, 64], 8, 2, 128, 7, masked=_some, train=False)
    _run(ps, dtype, [1, 7], [2500, 700], 4, 1, 40, 8, causal=True)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("group", [1, 3, 8])
def test_attention_wide_bias(ps, dtype, group):
    """The largest tables: many buckets, and distances at the limit of the group's span."""
    distance = (3080 // group - 129) // 2
    _run(ps, dtype, [260, 40], [260, 40], group, 1, 32, 9, buckets=128, distance=distance)
    _run(ps, dtype, [200], [200], group, 1, 64, 10, True, 64, 50)


def _strided(t, how):
    tokens, heads, d = t.shape
    if how == "heads first":
        s = torch.zeros(heads, tokens, d, dtype=t.dtype).cuda()
        v = s.transpose(0, 1)
    elif how == "padded":
        s = torch.full((tokens, heads + 1, d + 8), math.nan, dtype=t.dtype).cuda()
        v = s[:, :heads, :d]
    elif how == "odd start":
        s = torch.zeros(tokens * (heads * d + 1) + 3, dtype=t.dtype).cuda()
        v = s[3:].as_strided(t.shape, (heads * d + 1, d, 1), 3)
    else:  # values apart
        s = torch.zeros(tokens, heads, d, 2, dtype=t.dtype).cuda()
        v = s[..., 0]
    v.copy_(t)
    return v


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("how", ["heads first", "padded", "odd start", "apart"])
def test_attention_strides(ps, dtype, how):
    dt, rnd = DTYPES[dtype], _rnd(11)
    lens = [70, 20]
    o = _offsets(lens)
    q, k, v = rnd(90, 4, 64).to(dt), rnd(90, 2, 64).to(dt), rnd(90, 2, 64).to(dt)
    dout = rnd(90, 4, 64).to(dt)
    plan = ps.AttentionPlan(o, heads=4, kv_heads=2, head_dim=64, dtype=dt)
    s = [_strided(t, how) for t in (q, k, v, dout)]
    out, lse = plan.forward(*s[:3])
    val, tol = attention(q, k, v, o, o, dout=dout)
    check("out", out, val["out"], tol["out"])
    grads = plan.backward(s[3], *s[:3], _strided(out.cpu(), how), lse)
    for name, g in zip(("dq", "dk", "dv"), grads):
        check(name, g, val[name], tol[name])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_attention_expanded_values(ps, dtype):
    """Keys and values that are one token's, expanded: tokens 0 apart."""
    dt, rnd = DTYPES[dtype], _rnd(12)
    o = _offsets([40])
    q, k = rnd(40, 2, 32).to(dt), rnd(1, 2, 32).to(dt).expand(40, 2, 32)
    v = rnd(1, 2, 32).to(dt).expand(40, 2, 32)
    plan = ps.AttentionPlan(o, heads=2, head_dim=32, dtype=dt)
    out, lse = plan.forward(q.cuda(), k[:1].cuda().expand(40, 2, 32),
                            v[:1].cuda().expand(40, 2, 32))
    val, tol = attention(q, k, v, o, o)
    check("out", out, val["out"], tol["out"])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_attention_fused_projection(ps, dtype):
    _run(ps, dtype, [100, 3], [100, 3], 3, 3, 64, 13, fused=True, buckets=32, distance=128)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_attention_peaked_and_large_scores(ps, dtype):
    """Scores far from 0, of one size and of very different sizes; a scale of its own."""
    _run(ps, dtype, [90], [90], 2, 2, 64, 14, scale=1.0, spread=2.5)
    _run(ps, dtype, [90], [90], 2, 1, 64, 15, scale=0.01, buckets=8, distance=30,
         table=lambda b: b * 0 - 60000.0 if dtype != "f32" else b - 1e6)
    _run(ps, dtype, [90], [90], 2, 1, 64, 16, buckets=8, distance=30, causal=True,
         table=lambda b: b * 40)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("lowest", [False, True])
def test_attention_buckets_that_forbid(ps, dtype, lowest):
    """-infinity, and the type's lowest value, in buckets of the bias."""
    dt = DTYPES[dtype]
    value = torch.finfo(dt).min if lowest else -math.inf

    def table(b):
        b = b.clone()
        b[2:4] = value
        if not lowest:
            b[:, 1] = value  # a head that sees nothing
        return b

    if lowest:
        # rows keep keys of ordinary buckets: the lowest value only takes its own keys out
        got, (q, k, v, qo, ko, dout, bias, _) = _run(ps, dtype, [60], [60], 2, 2, 32, 17,
                                                     buckets=8, distance=30, table=table, odd=True)
        off = bias.clone().double()
        off[2:4] = -math.inf
        val, tol = attention(q, k, v, qo, ko, bias=off.to(dt), distance=30, dout=dout)
        for name in ("out", "dq", "dk", "dv"):
            check(name, got[name], val[name], tol[name] + 1e-30)
        return
    got, (q, k, v, qo, ko, dout, bias, _) = _run(ps, dtype, [60], [60], 2, 2, 32, 17, buckets=8,
                                                 distance=30, table=table, odd=True)
    assert not got["out"][:, 1].any() and torch.isneginf(got["lse"][:, 1]).all()
    for name in ("dq", "dk", "dv"):
        assert not got[name][:, 1].any()
    assert not got["dbias"][:, 1].any() and torch.isfinite(got["dbias"]).all()
    val, tol = attention(q[:, :1], k[:, :1], v[:, :1], qo, ko, bias=bias[:, :1], distance=30,
                         dout=dout[:, :1])
    for name in ("out", "dq", "dk", "dv"):
        check(name, got[name][:, :1], val[name], tol[name] + 1e-30)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("heads, kv_heads, d", [(2, 2, 64), (4, 1, 128), (3, 1, 20)])
@pytest.mark.parametrize("buckets", [0, 8])
def test_attention_causal_later_values_do_not_reach_back(ps, dtype, heads, kv_heads, d, buckets):
    """NaN and infinities in a document's tail: the rows before it are as without it."""
    dt, rnd = DTYPES[dtype], _rnd(18)
    lens, cut = [150, 20, 400], [101, 20, 333]
    o = _offsets(lens)
    n = int(o[-1])
    q, k, v = rnd(n, heads, d).to(dt), rnd(n, kv_heads, d).to(dt), rnd(n, kv_heads, d).to(dt)
    bias = rnd(buckets, heads).to(dt) if buckets else None
    keep = torch.zeros(n, dtype=torch.bool)
    for s in range(3):
        keep[int(o[s]):int(o[s]) + cut[s]] = True
    k[~keep], v[~keep], q[~keep] = math.nan, math.inf, math.nan
    plan = ps.AttentionPlan(o, heads=heads, kv_heads=kv_heads, head_dim=d, dtype=dt, causal=True,
                            num_buckets=buckets, max_distance=30 if buckets else 0)
    b = None if bias is None else bias.cuda()
    out, lse = plan.forward(q.cuda(), k.cuda(), v.cuda(), bias=b)
    small = _offsets(cut)
    dout = rnd(n, heads, d).to(dt)
    dq = plan.backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse, bias=b)[0]
    val, tol = attention(q[keep], k[keep], v[keep], small, small, True, bias=bias, distance=30,
                         dout=dout[keep])
    check("out", out.cpu()[keep], val["out"], tol["out"])
    check("lse", lse.cpu()[keep], val["lse"], tol["lse"])
    check("dq", dq.cpu()[keep], val["dq"], tol["dq"])


def test_attention_one_key_that_is_not_a_number(ps):
    """Without a mask it belongs to every row that sees it, and to no other sequence."""
    rnd = _rnd(19)
    o = _offsets([30, 30])
    q, k, v = rnd(60, 2, 64).half(), rnd(60, 2, 64).half(), rnd(60, 2, 64).half()
    v[40, 0, 3] = math.nan
    plan = ps.AttentionPlan(o, heads=2, head_dim=64, dtype=torch.float16)
    out = plan.forward(q.cuda(), k.cuda(), v.cuda())[0].cpu()
    assert torch.isfinite(out[:30]).all() and torch.isfinite(out[30:, 1]).all()
    assert torch.isnan(out[30:, 0, 3]).all() and torch.isfinite(out[30:, 0, :3]).all()


@pytest.mark.parametrize("size", [1e-6, 1.0, 1e3])
def test_attention_half_precision_gradients_of_any_size(ps, size):
    """binary16: small and large gradients keep their relative precision."""
    rnd = _rnd(20)
    o = _offsets([200, 33])
    q, k, v = rnd(233, 2, 64).half(), rnd(233, 2, 64).half(), rnd(233, 2, 64).half()
    dout = (rnd(233, 2, 64) * size).half()
    plan = ps.AttentionPlan(o, heads=2, head_dim=64, dtype=torch.float16)
    out, lse = plan.forward(q.cuda(), k.cuda(), v.cuda())
    got = plan.backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse)
    val, tol = attention(q, k, v, o, o, dout=dout)
    for name, g in zip(("dq", "dk", "dv"), got):
        check(name, g, val[name], tol[name])


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradient_against_differences(ps, causal):
    """The directional derivative of the kernels' own forward pass, from central differences.

    The step's truncation error is the oracle's at the same step; the rounding of the two sums is
    at most 2 E (values) / (2 step) of what they add up."""
    rnd = _rnd(21)
    o = _offsets([60, 9])
    base = {"q": rnd(69, 4, 32), "k": rnd(69, 2, 32), "v": rnd(69, 2, 32), "bias": rnd(8, 4)}
    dout = rnd(69, 4, 32)
    plan = ps.AttentionPlan(o, heads=4, kv_heads=2, head_dim=32, dtype=torch.float32,
                            causal=causal, num_buckets=8, max_distance=20)
    c = {n: t.cuda() for n, t in base.items()}
    out, lse = plan.forward(c["q"], c["k"], c["v"], bias=c["bias"])
    grads = dict(zip(("q", "k", "v", "bias"), plan.backward(dout.cuda(), c["q"], c["k"], c["v"],
                                                            out, lse, bias=c["bias"])))
    step = 2.0 ** -6
    for name in base:
        way = rnd(*base[name].shape)

        def at(s):
            return {n: (t + s * step * way if n == name else t) for n, t in base.items()}

        def gpu(s):
            t = {n: x.cuda() for n, x in at(s).items()}
            return float((plan.forward(t["q"], t["k"], t["v"], bias=t["bias"])[0].double().cpu() *
                          dout.double()).sum())

        def oracle(s):
            t = at(s)
            val, tol = attention(t["q"], t["k"], t["v"], o, o, causal, None, None, t["bias"], 20)
            return float((val["out"] * dout.double()).sum()), \
                float((tol["out"] * dout.double().abs()).sum())

        (hi, hi_tol), (lo, lo_tol) = oracle(1), oracle(-1)
        val, tol = attention(base["q"], base["k"], base["v"], o, o, causal, None, None,
                             base["bias"], 20, dout)
        exact = float((val["d" + name] * way.double()).sum())
        truncation = abs((hi - lo) / (2 * step) - exact)
        got = float((grads[name].double().cpu() * way.double()).sum())
        grad_tol = float((tol["d" + name] * way.double().abs()).sum())
        assert abs((gpu(1) - gpu(-1)) / (2 * step) - got) <= \
            truncation + (hi_tol + lo_tol) / (2 * step) + grad_tol


def test_attention_autograd_and_streams(ps):
    rnd = _rnd(22)
    o = _offsets([40, 25])
    plan = ps.AttentionPlan(o, heads=2, head_dim=32, dtype=torch.float32, num_buckets=8,
                            max_distance=20)
    base = [rnd(65, 2, 32), rnd(65, 2, 32), rnd(65, 2, 32), rnd(8, 2)]
    t = [x.cuda().requires_grad_() for x in base]
    out = ps.attention(t[0], t[1], t[2], plan, bias=t[3])
    dout = rnd(65, 2, 32)
    out.backward(dout.cuda())
    val, tol = attention(*base[:3], o, o, bias=base[3], distance=20, dout=dout)
    check("out", out, val["out"], tol["out"])
    for name, x in zip(("dq", "dk", "dv", "dbias"), t):
        check(name, x.grad, val[name], tol[name])
    # another stream than the current one, work queued behind a copy on it
    s = torch.cuda.Stream()
    c = [x.detach() for x in t]
    s.wait_stream(torch.cuda.current_stream())
    got, lse = plan.forward(*c[:3], bias=c[3], stream=s)
    grads = plan.backward(dout.cuda(), *c[:3], got, lse, bias=c[3], stream=s)
    s.synchronize()
    check("out", got, val["out"], tol["out"])
    check("dq", grads[0], val["dq"], tol["dq"])


def test_operators_in_a_graph(ps):
    """Captured once, replayed on new inputs with eager work in between."""
    rnd = _rnd(23)
    o = _offsets([300, 41, 7])
    n = 348
    plan = ps.AttentionPlan(o, heads=4, kv_heads=2, head_dim=64, dtype=torch.bfloat16,
                            num_buckets=32, max_distance=128, causal=True)
    x = [rnd(n, 4, 64).bfloat16().cuda(), rnd(n, 2, 64).bfloat16().cuda(),
         rnd(n, 2, 64).bfloat16().cuda(), rnd(n, 4, 64).bfloat16().cuda()]
    bias, w = rnd(32, 4).bfloat16().cuda(), rnd(256).bfloat16().cuda()

    def step():
        out, lse = plan.forward(*x[:3], bias=bias)
        y, h, mean, rstd = ps.layer_norm_forward(out.reshape(n, 256), w, w)
        dx, dw, db = ps.layer_norm_backward(x[3].reshape(n, 256), h, w, mean, rstd)
        return (y, dw, db) + plan.backward(dx.reshape(n, 4, 64), *x[:3], out, lse, bias=bias)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        for t in x:
            t.copy_(rnd(*t.shape).bfloat16())
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), i


def test_attention_refusals(ps):
    o = _offsets([4])
    kw = dict(heads=2, head_dim=8, dtype=torch.float32)
    for bad in (dict(q_offsets=torch.tensor([0.0, 4.0])), dict(q_offsets=torch.zeros(0).long()),
                dict(k_offsets=_offsets([1, 3])), dict(head_dim=0), dict(device="cpu")):
        with pytest.raises(ValueError):
            ps.AttentionPlan(**{**dict(q_offsets=o), **kw, **bad})
    with pytest.raises(TypeError):
        ps.AttentionPlan(o, heads=2, head_dim=8, dtype=torch.float64)
    for bad in (dict(head_dim=129), dict(kv_heads=3), dict(scale=-1.0),
                dict(num_buckets=32, max_distance=4)):
        with pytest.raises(ps.SieveError):
            ps.AttentionPlan(o, **{**kw, **bad})
    with pytest.raises(ps.SieveError):
        ps.AttentionPlan(torch.tensor([0, 5, 2]), **kw)
    plan = ps.AttentionPlan(o, **kw)
    x = torch.zeros(4, 2, 8).cuda()
    with pytest.raises(TypeError):
        plan.forward(x.half(), x, x)
    for args in ((x[:3], x, x), (x, x[:, :1], x), (x, x, x.cpu())):
        with pytest.raises(ValueError):
            plan.forward(*args)
    with pytest.raises(ValueError):
        plan.forward(x, x, x, key_mask=torch.ones(3, dtype=torch.bool).cuda())
    with pytest.raises(ValueError):
        plan.forward(x, x, x, bias=torch.zeros(4, 2).cuda())
    out, lse = plan.forward(x, x, x)
    with pytest.raises(ValueError):
        plan.backward(x, x, x, x, out, lse[:2])
    plan.close()
    with pytest.raises(ps.SieveError):
        plan.forward(x, x, x)


def test_bucket_definition(ps):
    """The table's edges as the kernels see them: a bias that names its bucket, one query."""
    for causal in (False, True):
        n = 300
        plan = ps.AttentionPlan([0, n], [0, n], heads=1, head_dim=1, dtype=torch.float32,
                                causal=causal, num_buckets=32, max_distance=128)
        # uniform scores but for the bucket asked about: its share of the keys
        zero = torch.zeros(n, 1, 1).cuda()
        for b in range(0, 32, 5):
            bias = torch.zeros(32, 1)
            bias[b] = -math.inf
            _, lse = plan.forward(zero, zero, zero, bias=bias.cuda())
            for i in (0, 1, 150, n - 1):
                keys = range(i + 1) if causal else range(n)
                left = sum(bucket(j - i, 32, 128, causal) != b for j in keys)
                want = math.log(left) if left else -math.inf
                assert abs(float(lse[i, 0]) - want) < 1e-5 or float(lse[i, 0]) == want
