"""Layer norm and packed attention in 64 bits on the CPU, with bounds on how far a computation
in a given type may be from them.

The bounds follow the operations: products and sums in fp32 (unit roundoff E), values rounded to
the inputs' type (unit roundoff u) where the operators round them, that is the outputs, and the
probabilities and dS in front of the second matrix products.  They are worked out for every
value from the magnitudes that enter it."""
import math

import torch

E = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
#: smallest step of the type (what a value below its normal range may be off by, twice over)
TINY = {torch.float32: 2.0 ** -148, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -132}


def bucket(rel, buckets, distance, causal):
    """Bucket of a relative position, in whole numbers."""
    side = buckets if causal else buckets // 2
    base = side if rel > 0 and not causal else 0
    m = max(-rel, 0) if causal else abs(rel)
    exact = side // 2
    if m < exact:
        return base + m
    if m >= distance:
        return base + side - 1
    k = side - exact
    # floor(k log(m / exact) / log(distance / exact)): the largest j with
    # (m / exact)^k >= (distance / exact)^j
    j = sum(m ** k * exact ** i >= distance ** i * exact ** k for i in range(1, k + 1))
    return base + min(exact + j, side - 1)


def norm(x, weight, bias, eps, residual=None, dy=None, dh=None):
    """({name: value}, {name: bound}) of the forward pass, and of the backward pass with dy."""
    u, n, dt = UNIT[x.dtype], x.shape[-1], x.dtype
    uw = UNIT[weight.dtype]
    h = x.double()
    if residual is not None:
        h = (x.float() + residual.float()).to(dt).double()  # fp32 adds two such values exactly
    h = h.reshape(-1, n)
    w = weight.double()
    b = torch.zeros(n, dtype=torch.float64) if bias is None else bias.double()
    mean = h.mean(1, keepdim=True)
    c = h - mean
    var = c.square().mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    unit = c * rstd
    y = unit * w + b
    # a sum of n terms in fp32, at most ceil(n / 64) + 8 in a row of additions
    s = (math.ceil(n / 64) + 12) * E
    d_mean = s * h.abs().mean(1, keepdim=True)
    # the variance from differences that are off by d_mean and their own rounding
    d_var = (2 * s + 4 * E) * var + 2 * d_mean * c.abs().mean(1, keepdim=True) + d_mean ** 2
    r_rstd = 0.5 * d_var / (var + eps) + 8 * E  # relative
    d_unit = rstd * (d_mean + E * h.abs()) + unit.abs() * (r_rstd + 4 * E)
    val = {"h": h, "y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    tol = {"y": d_unit * w.abs() + (u + 4 * E) * (y.abs() + (unit * w).abs()) + TINY[dt],
           "mean": d_mean[:, 0] + 1e-30, "rstd": (r_rstd * rstd)[:, 0]}
    if dy is None:
        return val, tol
    dy = dy.double().reshape(-1, n)
    g = dy * w
    m1, m2 = g.mean(1, keepdim=True), (g * unit).mean(1, keepdim=True)
    dx = rstd * (g - m1 - unit * m2)
    ga, ua = g.abs(), unit.abs()
    d_m1 = (s + 2 * E) * ga.mean(1, keepdim=True)
    d_m2 = (s + 4 * E) * (ga * ua).mean(1, keepdim=True) + (ga * d_unit).mean(1, keepdim=True)
    d_dx = rstd * (d_m1 + ua * d_m2 + d_unit * m2.abs() + 8 * E * (ga + m1.abs() + ua * m2.abs()))
    d_dx = d_dx + (r_rstd + 4 * E) * dx.abs()
    if dh is not None:
        dh = dh.double().reshape(-1, n)
        dx = dx + dh
        d_dx = d_dx + 2 * E * dh.abs()
    rows = h.shape[0]
    # sums over rows: a thread's rows, the waves and the partial rows one after another
    sr = (math.ceil(rows / 4) + 64) * E
    val.update(dx=dx, dweight=(dy * unit).sum(0), dbias=dy.sum(0))
    tol.update(dx=d_dx + u * dx.abs() + TINY[dt],
               dweight=(sr + 4 * E) * (dy * unit).abs().sum(0) + (dy.abs() * d_unit).sum(0) +
               uw * val["dweight"].abs() + TINY[weight.dtype],
               dbias=sr * dy.abs().sum(0) + uw * val["dbias"].abs() + TINY[weight.dtype])
    return val, tol


def attention(q, k, v, q_offsets, k_offsets, causal=False, scale=None, mask=None, bias=None,
              distance=0, dout=None):
    """({name: value}, {name: bound}) of out and lse, and with dout of dq, dk, dv and dbias."""
    dt, d = q.dtype, q.shape[2]
    u, tiny = UNIT[dt], TINY[dt]
    heads, kv_heads = q.shape[1], k.shape[1]
    group = heads // kv_heads
    scale = 1 / math.sqrt(d) if scale is None else scale
    Q, K, V = q.double(), k.double(), v.double()
    names = ["out"] + (["dq", "dk", "dv"] if dout is not None else [])
    like = {"out": Q, "dq": Q, "dk": K, "dv": K}
    val = {n: torch.zeros_like(like[n]) for n in names}
    tol = {n: torch.zeros_like(like[n]) for n in names}
    val["lse"] = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    tol["lse"] = torch.zeros(q.shape[:2], dtype=torch.float64)
    if bias is not None and dout is not None:
        val["dbias"] = torch.zeros(bias.shape, dtype=torch.float64)
        tol["dbias"] = torch.zeros(bias.shape, dtype=torch.float64)
    for s in range(len(q_offsets) - 1):
        q0, q1, k0, k1 = (int(x) for x in (q_offsets[s], q_offsets[s + 1], k_offsets[s],
                                           k_offsets[s + 1]))
        m, n = q1 - q0, k1 - k0
        if m == 0 or n == 0:
            continue
        rel = torch.arange(n)[None, :] - (torch.arange(m) + n - m)[:, None]
        seen = torch.ones(m, n, dtype=torch.bool)
        keep = torch.ones(n, dtype=torch.bool)
        if mask is not None:
            keep = mask[k0:k1].bool()
            seen = seen & keep[None, :]
        if causal:
            seen = seen & (rel <= 0)
        if bias is not None:
            reach = range(-(n + m), n + m + 1)
            of = torch.tensor([bucket(r, bias.shape[0], distance, causal) for r in reach])
            which = of[rel + (n + m)]
        pairs = seen
        for h in range(heads):
            g = h // group
            seen = pairs  # and no bias of -infinity
            if bias is not None:
                seen = seen & (bias[:, h].double()[which] != -math.inf)
            some = seen.any(1)
            qi, ki, vi = Q[q0:q1, h], K[k0:k1, g].clone(), V[k0:k1, g].clone()
            ki[~keep], vi[~keep] = 0, 0
            sc, mag = scale * (qi @ ki.T), scale * (qi.abs() @ ki.abs().T)
            if bias is not None:
                add = torch.where(seen, bias[:, h].double()[which], 0.0)
                sc, mag = sc + add, mag + add.abs()
            sc = torch.where(seen, sc, -math.inf)
            lse = torch.logsumexp(sc, 1)
            p = torch.where(seen & some[:, None], torch.exp(sc - lse[:, None]), 0.0)
            o = p @ vi
            # a score's error: the product's terms, scaling, the bias and the exponent's argument
            mag = torch.where(seen, mag, 0.0)
            ds_ = (d + 8) * E * mag
            worst = ds_.amax(1) + 8 * E * (1 + torch.where(some, lse, 0.0).abs() + mag.amax(1))
            rp = 2 * worst + 8 * E  # relative error of a probability, before it is rounded
            acc = (n / 8 + 16) * E  # a sum over keys
            ov = p @ vi.abs()
            # probabilities rounded for the product, their sum likewise or not
            d_o = (2 * u + 2 * rp + 2 * acc)[:, None] * ov + u * o.abs() + tiny
            # a key whose probability falls below the type's normal range (binary16, scaled up)
            d_o = d_o + 2.0 ** -34 * p.amax(1, keepdim=True) * vi.abs().sum(0) * (u > E)
            val["out"][q0:q1, h], tol["out"][q0:q1, h] = o, d_o
            val["lse"][q0:q1, h] = lse
            tol["lse"][q0:q1, h] = torch.where(some, worst + u * (u > E) + acc + 4 * E, 0.0)
            if dout is None:
                continue
            do = dout[q0:q1, h].double().clone()
            do[~some] = 0
            dp = do @ vi.T
            di = (do * o).sum(1, keepdim=True)
            ds = p * (dp - di)
            d_dp = (d + 4) * E * (do.abs() @ vi.abs().T)
            d_di = (do.abs() * d_o).sum(1, keepdim=True) + \
                (d + 4) * E * (do.abs() * o.abs()).sum(1, keepdim=True)
            # dS before it is rounded, and rounded (binary16 below its normal range: scaled so
            # that the largest of the sequence is at 2^13)
            d_ds = ds.abs() * (rp[:, None] + 8 * E) + p * (d_dp + d_di) * (1 + rp[:, None])
            d_dsr = d_ds + u * (ds.abs() + d_ds) + 2.0 ** -37 * ds.abs().amax() * (u > E)
            val["dq"][q0:q1, h] = scale * (ds @ ki)
            tol["dq"][q0:q1, h] = scale * ((d_dsr + acc * ds.abs()) @ ki.abs()) + tiny + \
                (u + 4 * E) * val["dq"][q0:q1, h].abs()
            accq = (m * group / 8 + 16) * E  # a sum over queries
            # the group's heads add up in the accumulator: rounded once
            d_p = p * (u + rp[:, None]) + 2.0 ** -38 * (u > E) * seen
            val["dk"][k0:k1, g] += scale * (ds.T @ qi)
            val["dv"][k0:k1, g] += p.T @ do
            tol["dk"][k0:k1, g] += scale * ((d_dsr + accq * ds.abs()).T @ qi.abs())
            tol["dv"][k0:k1, g] += (d_p + accq * p).T @ do.abs()
            if bias is not None:
                accb = (m + n + 64) * E
                for name, x in (("v", ds), ("t", d_ds + accb * ds.abs())):
                    to = (val if name == "v" else tol)["dbias"][:, h]
                    to.index_add_(0, which.reshape(-1), torch.where(seen, x, 0.0).reshape(-1))
    if dout is not None:
        for name in ("dk", "dv"):
            tol[name] += (u + 4 * E) * val[name].abs() + tiny
    if "dbias" in val:
        tol["dbias"] += u * val["dbias"].abs() + tiny
    return val, tol


def check(name, got, want, tol):
    """Every value within its bound; what is not finite is the same."""
    got = got.detach().double().cpu().reshape(want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), name
    assert torch.equal(got[~fine], want[~fine]), name
    far = (got - want).abs()[fine] - tol[fine]
    assert far.numel() == 0 or float(far.max()) <= 0, \
        f"{name}: {int((far > 0).sum())} of {far.numel()} values past their bound, the worst by " \
        f"{float(far.max()):.3g} over {float(tol[fine][far.argmax()]):.3g}"
