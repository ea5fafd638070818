"""Performance cases of the text-encoder operators.

The vectors that the index searches are written by a text encoder over a packed batch of
documents; these are the encoder's own operators, for embedding a corpus and for training the
encoder on near-duplicate pairs.

Every case is a dict of plain values.  ``op`` is

  "norm"    layer norm over the last axis of [rows, n], with an added residual where asked
            (h = x + residual, y = norm(h)); with ``train`` the gradients too
  "attend"  attention over packed documents of lo..hi tokens (the lengths follow from the case):
            ``heads`` query heads share ``kv_heads`` key heads of ``d`` values; ``queries`` = 0
            attends from every token of a document, else from that many queries per document
            that stand at its end; ``buckets`` > 0 adds a learned bias by buckets of the relative
            position up to ``distance``; ``masked`` is the share of keys that the key mask leaves
            out (their keys and values are not numbers); ``fused`` keeps q, k and v in one
            projection's output; with ``train`` the gradients too
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


def _norm(name, rows, n, dtype, wdtype, residual, train):
    c = dict(op="norm", rows=rows, n=n, dtype=dtype, wdtype=wdtype, residual=residual, train=train)
    return dict(c, name=name) if name else c


def _attend(name, docs, lo, hi, heads, kv_heads, d, dtype, *, queries=0, causal=False, buckets=0,
            distance=0, masked=0.0, fused=False, train=False):
    c = dict(op="attend", docs=docs, lo=lo, hi=hi, heads=heads, kv_heads=kv_heads, d=d,
             dtype=dtype, queries=queries, causal=causal, buckets=buckets, distance=distance,
             masked=masked, fused=fused, train=train)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short text embedded at ingest: launches and latency
        _norm("norm_one_text_24x768_f16", 24, 768, "f16", "f16", True, False),
        # a large corpus batch embedded at the width of the 768-dimension index
        _norm("norm_corpus_262144x768_f16", 262144, 768, "f16", "f16", True, False),
        # a training batch with weights kept in 32 bits
        _norm("norm_train_65536x1024_bf16", 65536, 1024, "bf16", "f32", True, True),
        # a ragged token count and a width that is no multiple of a vector load
        _norm("norm_train_20001x515_f32", 20001, 515, "f32", "f32", False, True),
        # the same short text's attention
        _attend("attend_one_text_24_12x64_f16", 1, 24, 24, 12, 12, 64, "f16", buckets=32,
                distance=128, fused=True),
        # a corpus batch of ragged documents, relative position bias, fused projection
        _attend("attend_corpus_512docs_12x64_f16", 512, 16, 512, 12, 12, 64, "f16", buckets=32,
                distance=128, fused=True),
        # one pooling query per long document: key and value reads
        _attend("attend_pool_32docs_16x128_bf16", 32, 1000, 30000, 16, 4, 128, "bf16", queries=1),
        # one long document in an encoder taken from a causal model, shared key heads
        _attend("attend_long_12007_16x128_bf16", 1, 12007, 12007, 16, 4, 128, "bf16", causal=True),
        # a handful of short pairs: the smallest training step
        _attend("attend_train_pairs_8docs_12x64_bf16", 8, 5, 60, 12, 12, 64, "bf16", buckets=32,
                distance=128, train=True),
        # a contrastive batch of ragged documents with the bias table's gradient
        _attend("attend_train_256docs_12x64_f16", 256, 16, 512, 12, 12, 64, "f16", buckets=32,
                distance=128, fused=True, train=True),
        # long causal documents in training, shared key heads
        _attend("attend_train_long_2docs_16x128_bf16", 2, 5000, 6100, 16, 4, 128, "bf16",
                causal=True, train=True),
        # 32-bit training of a small encoder: an odd head size, masked tokens, whole documents
        # masked among them
        _attend("attend_train_masked_100docs_8x40_f32", 100, 1, 300, 8, 8, 40, "f32", buckets=16,
                distance=64, masked=0.15, train=True),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "texts", "texts_train", "long", "long_train", "pool"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    if kind.startswith("norm"):
        n = rng.choice([64, 128, 384, 512, 515, 768, 1024, 1000, 2048, 4096, 77])
        train = kind == "norm_train"
        most = 2 ** 25 if train or dtype == "f32" else 2 ** 26
        rows = max(1, min(_log(rng, 16, 262144), most // n))
        return _norm(None, rows, n, dtype, rng.choice([dtype, "f32"]), rng.random() < 0.5, train)
    d = rng.choice([32, 40, 64, 64, 64, 80, 96, 128])
    kv = rng.choice([2, 4, 8, 12])
    heads = min(16, kv * rng.choice([1, 1, 2, 4])) if kv < 12 else kv
    train = kind.endswith("train")
    if kind == "pool":
        hi = _log(rng, 200, 30000)
        docs = max(1, min(_log(rng, 1, 200), 2 ** 31 // (hi * heads * d * 4)))
        return _attend(None, docs, max(1, hi // 20), hi, heads, kv, d, dtype,
                       queries=rng.choice([1, 1, 2, 5]), masked=rng.choice([0.0, 0.1]))
    if kind.startswith("long"):
        hi = _log(rng, 700, 2500 if dtype == "f32" else 5000)
        nb = rng.choice([0, 0, 32])
        return _attend(None, rng.choice([1, 2, 3]) if hi < 2500 else 1, hi * 3 // 4, hi, heads, kv,
                       d, dtype, causal=rng.random() < 0.6, buckets=nb, distance=4 * nb,
                       train=train)
    hi = _log(rng, 8, 512)
    docs = max(1, min(_log(rng, 1, 512), 2 ** 30 // (hi * hi * heads * (2 if train else 1))))
    nb = rng.choice([0, 16, 32, 32])
    fused = heads == kv and heads * d != 1024 and rng.random() < 0.5
    return _attend(None, docs, max(1, hi // 30), hi, heads, kv, d, dtype,
                   causal=rng.random() < 0.25, buckets=nb, distance=4 * nb,
                   masked=rng.choice([0.0, 0.0, 0.15]), fused=fused, train=train)


def _lengths(c):
    """Tokens of each document: a function of the case alone."""
    r = random.Random("%d %d %d" % (c["docs"], c["lo"], c["hi"]))
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["docs"])]


def _pairs(c):
    """(query, key) pairs of one head that the causal rule leaves."""
    total = 0
    for n in _lengths(c):
        m = c["queries"] or n
        total += m * n - (m * (m - 1) // 2 if c["causal"] else 0)
    return total


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "norm":
        grid = c["rows"] * c["n"]
        forward = grid * size * (4 if c["residual"] else 2)
        backward = grid * size * 3 if c["train"] else 0
        return {"bytes": forward + backward, "flops": grid * (20 if c["train"] else 8)}
    keys = sum(_lengths(c))
    rows = c["docs"] * c["queries"] if c["queries"] else keys
    io_q, io_k = rows * c["heads"] * c["d"] * size, keys * c["kv_heads"] * c["d"] * size
    pairs = _pairs(c) * c["heads"] * c["d"]
    if not c["train"]:
        return {"bytes": 2 * io_q + 2 * io_k, "flops": 4 * pairs}
    # forward: q, k, v read, the output written; backward: q, k, v, the output and its gradient
    # read, three gradients written
    return {"bytes": 2 * io_q + 2 * io_k + 4 * io_q + 4 * io_k, "flops": 14 * pairs}


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def prepare(case, seed):
    c, dev = case, _device()
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 11)
    dt = DTYPES[c["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(shape, generator=g, device=dev) * scale).to(dtype)

    if c["op"] == "norm":
        wt = DTYPES[c["wdtype"]]
        n = c["n"]
        # activations of a trained encoder: a few channels much larger than the rest
        channel = torch.exp(0.6 * torch.randn(n, generator=g, device=dev))
        s = {"case": c, "x": (normal(c["rows"], n, dtype=torch.float32) * channel + 0.1).to(dt),
             "weight": normal(n, scale=0.2, dtype=wt) + 1, "bias": normal(n, scale=0.1, dtype=wt)}
        s["residual"] = normal(c["rows"], n, scale=2.0) if c["residual"] else None
        if c["train"]:
            s["dy"] = normal(c["rows"], n, scale=0.05)
        return s
    lens = _lengths(c)
    keys = sum(lens)
    qlens = [c["queries"]] * len(lens) if c["queries"] else lens
    rows, h, hk, d = sum(qlens), c["heads"], c["kv_heads"], c["d"]
    s = {"case": c}
    if c["fused"]:
        qkv = normal(keys, 3, h, d)
        qkv[:, :2] *= 1.3
        s["q"], s["k"], s["v"] = qkv[:, 0], qkv[:, 1], qkv[:, 2]
    else:
        s["q"] = normal(rows, h, d, scale=1.3)
        s["k"], s["v"] = normal(keys, hk, d, scale=1.3), normal(keys, hk, d)
    s["bias"] = normal(c["buckets"], h, scale=0.7) if c["buckets"] else None
    s["mask"] = None
    if c["masked"]:
        keep = torch.rand(keys, generator=g, device=dev) >= c["masked"]
        start = 0
        for i, n in enumerate(lens):
            if i % 11 == 5:
                keep[start:start + n] = False
            start += n
        s["mask"] = keep
        s["k"][~keep] = math.nan
        s["v"][~keep] = math.nan
    if c["train"]:
        s["dout"] = normal(rows, h, d, scale=0.1)
    # where each document's rows lie in a padded batch, and back
    off = lambda v: torch.tensor([0] + v, dtype=torch.int64).cumsum(0)  # noqa: E731
    s["q_offsets"], s["k_offsets"] = off(qlens), off(lens)
    if own:
        import paper_2608_03199_amd as ps
        s["plan"] = ps.AttentionPlan(s["q_offsets"], s["k_offsets"], heads=h, kv_heads=hk,
                                     head_dim=d, dtype=dt, causal=c["causal"],
                                     num_buckets=c["buckets"], max_distance=c["distance"])
    else:
        ql, kl = torch.tensor(qlens, device=dev), torch.tensor(lens, device=dev)
        for name, ln, o in (("q", ql, s["q_offsets"]), ("k", kl, s["k_offsets"])):
            at = torch.arange(int(ln.max()), device=dev)
            live = at[None, :] < ln[:, None]
            s[name + "_live"] = live
            s[name + "_index"] = torch.where(live, o[:-1].to(dev)[:, None] + at[None, :], 0)
        if c["buckets"]:
            s["bucket_of"] = torch.tensor(_buckets(max(lens), c), device=dev)
    return s


def _bucket(rel, buckets, distance, causal):
    """Bucket of a relative position (key minus query): exact up to half of a side's buckets,
    then logarithmic up to the distance.  Whole numbers only, so that no edge is rounded."""
    side = buckets if causal else buckets // 2
    base = side if rel > 0 and not causal else 0
    n = max(-rel, 0) if causal else abs(rel)
    exact = side // 2
    if n < exact:
        return base + n
    if n >= distance:
        return base + side - 1
    steps = side - exact
    up = sum(n ** steps * exact ** j >= distance ** j * exact ** steps for j in range(1, steps))
    return base + exact + up


def _buckets(longest, c):
    """Buckets of the relative positions -(longest - 1) .. longest - 1."""
    near = {r: _bucket(r, c["buckets"], c["distance"], c["causal"])
            for r in range(-c["distance"], c["distance"] + 1)}
    return [near[max(-c["distance"], min(c["distance"], r))] for r in range(1 - longest, longest)]


def run(state):
    c = state["case"]
    if own:
        return _run_norm_own(state, c) if c["op"] == "norm" else _run_attend_own(state, c)
    return _run_norm_plain(state, c) if c["op"] == "norm" else _run_attend_plain(state, c)


def _run_norm_own(s, c):
    import paper_2608_03199_amd as ps
    y, h, mean, rstd = ps.layer_norm_forward(s["x"], s["weight"], s["bias"], EPS, s["residual"])
    out = {"y": y}
    if c["residual"]:
        out["h"] = h
    if c["train"]:
        out["dx"], out["dweight"], out["dbias"] = ps.layer_norm_backward(
            s["dy"], h, s["weight"], mean, rstd, bias_grad=True)
    return out


def _run_attend_own(s, c):
    out, lse = s["plan"].forward(s["q"], s["k"], s["v"], key_mask=s["mask"], bias=s["bias"])
    got = {"out": out}
    if c["train"]:
        got["dq"], got["dk"], got["dv"], dbias = s["plan"].backward(
            s["dout"], s["q"], s["k"], s["v"], out, lse, key_mask=s["mask"], bias=s["bias"])
        if c["buckets"]:
            got["dbias"] = dbias
    return got


def _run_norm_plain(s, c):
    h = s["x"].float()
    if c["residual"]:
        # the sum is kept in the activations' type, as the next layer reads it
        h = (h + s["residual"].float()).to(s["x"].dtype)
    out = {"h": h} if c["residual"] else {}
    h, w = h.float(), s["weight"].float()
    centred = h - h.mean(1, keepdim=True)
    rstd = (centred.square().mean(1, keepdim=True) + EPS).rsqrt()
    unit = centred * rstd
    out["y"] = (unit * w + s["bias"].float()).to(s["x"].dtype)
    if c["train"]:
        dy = s["dy"].float()
        du = dy * w
        dx = rstd * (du - du.mean(1, keepdim=True) - unit * (du * unit).mean(1, keepdim=True))
        out["dx"] = dx.to(s["x"].dtype)
        out["dweight"] = (dy * unit).sum(0).to(s["weight"].dtype)
        out["dbias"] = dy.sum(0).to(s["bias"].dtype)
    return out


def _run_attend_plain(s, c):
    dt, h, hk, d = s["q"].dtype, c["heads"], c["kv_heads"], c["d"]
    share, scale = h // hk, 1.0 / math.sqrt(d)
    q_live, k_live = s["q_live"], s["k_live"]
    docs, lq, lk = q_live.shape[0], q_live.shape[1], k_live.shape[1]

    def padded(x, index, live):  # [docs, heads, length, d]
        x = x.float()[index]
        return torch.where(live[:, :, None, None], x, 0.0).transpose(1, 2)

    keep = k_live if s["mask"] is None else k_live & s["mask"][s["k_index"]]
    q = padded(s["q"], s["q_index"], q_live)
    k = padded(s["k"], s["k_index"], keep).repeat_interleave(share, 1)
    v = padded(s["v"], s["k_index"], keep).repeat_interleave(share, 1)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    seen = keep[:, None, None, :] & q_live[:, None, :, None]
    shift = k_live.sum(1) - q_live.sum(1)  # queries stand at their document's end
    place = torch.arange(lq, device=q.device)[None, :] + shift[:, None]
    rel = torch.arange(lk, device=q.device)[None, None, :] - place[:, :, None]
    if c["causal"]:
        seen = seen & (rel <= 0)[:, None]
    if c["buckets"]:
        # self-attention: one table of positions for every document
        score += s["bias"].float()[s["bucket_of"][rel[:1] + (lk - 1)]].permute(0, 3, 1, 2)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(3, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    del score
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, v)
    got = {"out": o.transpose(1, 2)[q_live].to(dt)}
    if not c["train"]:
        return got
    do = padded(s["dout"], s["q_index"], q_live)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (do * o).sum(3, keepdim=True))
    del dp, p
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) * scale
    got["dq"] = dq.transpose(1, 2)[q_live].to(dt)
    for name, x in (("dk", dk), ("dv", dv)):
        x = x.reshape(docs, hk, share, lk, d).sum(2).transpose(1, 2)
        got[name] = torch.where(keep[:, :, None, None], x, 0.0)[k_live].to(dt)
    if c["buckets"]:
        # rows shifted against each other so that a relative position becomes a column
        near = ds.sum(0)
        near = torch.nn.functional.pad(near, (lq - 1, 0)).reshape(h, -1)
        near = torch.nn.functional.pad(near, (0, lq)).reshape(h, lq, lq + lk)
        diagonal = near.sum(1)[:, :-1]
        one = torch.nn.functional.one_hot(s["bucket_of"], c["buckets"]).float()
        got["dbias"] = torch.matmul(diagonal, one).t().contiguous().to(dt)
    return got


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "norm":
        return _exact_norm(s, c)
    return _exact_attend(s, c)


def _exact_norm(s, c):
    h = s["x"]
    if c["residual"]:
        h = (h.double() + s["residual"].double()).to(h.dtype)
    rows = h.shape[0]
    w = s["weight"].double().requires_grad_(c["train"])
    b = s["bias"].double().requires_grad_(c["train"])
    out = {"y": [], "dx": []}
    for at in range(0, rows, 32768):  # pieces of the rows, for memory
        x = h[at:at + 32768].double().requires_grad_(c["train"])
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        y = (x - mean) / torch.sqrt(var + EPS) * w + b
        if c["train"]:
            y.backward(s["dy"][at:at + 32768].double())
            out["dx"].append(x.grad)
        out["y"].append(y.detach())
    got = {"y": torch.cat(out["y"])}
    if c["residual"]:
        got["h"] = h.double()
    if c["train"]:
        got.update(dx=torch.cat(out["dx"]), dweight=w.grad, dbias=b.grad)
    return got


def _exact_attend(s, c):
    if _pairs(c) * c["heads"] * c["d"] > 2 ** 42:
        return None
    h, hk, d, train = c["heads"], c["kv_heads"], c["d"], c["train"]
    lens = _lengths(c)
    dev = s["q"].device
    q, k, v = (s[n].double() for n in "qkv")
    bias = s["bias"].double().requires_grad_(train) if c["buckets"] else None
    got = {"out": torch.zeros_like(q)}
    if train:
        got.update(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
    group = h // hk
    tables = {}
    k0 = q0 = 0
    for n in lens:
        m = c["queries"] or n
        rel = torch.arange(n, device=dev)[None, :] - (torch.arange(m, device=dev) + n - m)[:, None]
        keep = torch.ones(n, dtype=torch.bool, device=dev)
        if s["mask"] is not None:
            keep = s["mask"][k0:k0 + n]
        seen = keep[None, :].expand(m, n)
        if c["causal"]:
            seen = seen & (rel <= 0)
        some = seen.any(1)
        if bias is not None and n not in tables:
            tables[n] = torch.tensor(_buckets(n, c), device=dev)
        per = max(1, 2 ** 27 // (m * n))  # heads at a time, for memory
        for a in range(0, h, per):
            e = min(h, a + per)
            which = torch.arange(a, e, device=dev) // group
            x = [q[q0:q0 + m, a:e], k[k0:k0 + n][:, which], v[k0:k0 + n][:, which]]
            x = [t.transpose(0, 1).contiguous() for t in x]
            x[1], x[2] = (torch.where(keep[None, :, None], t, 0.0) for t in x[1:])
            x = [t.detach().requires_grad_(train) for t in x]
            sc = torch.bmm(x[0], x[1].transpose(1, 2).contiguous()) / math.sqrt(d)
            if bias is not None:
                sc = sc + bias[tables[n][rel + n - 1]][:, :, a:e].permute(2, 0, 1)
            sc = sc.masked_fill(~seen, -math.inf).masked_fill(~some[:, None], 0.0)
            pr = torch.softmax(sc, 2) * some[:, None]
            o = torch.bmm(pr, x[2])
            got["out"][q0:q0 + m, a:e] = o.detach().transpose(0, 1)
            if train:
                o.backward(s["dout"][q0:q0 + m, a:e].double().transpose(0, 1).contiguous())
                got["dq"][q0:q0 + m, a:e] = x[0].grad.transpose(0, 1)
                for name, t in (("dk", x[1]), ("dv", x[2])):
                    grad = t.grad * keep[None, :, None]
                    got[name][k0:k0 + n].index_add_(1, which, grad.transpose(0, 1))
        k0, q0 = k0 + n, q0 + m
    if train:
        got["dk"], got["dv"] = got["dk"].clone(), got["dv"].clone()
    if bias is not None and train:
        got["dbias"] = bias.grad
    return got
