"""Performance cases of the operators around a text encoder's blocks: the table at its input, the
loss at its output, and the update of the matrices between them.

Every case is a dict of plain values.  ``op`` is

  "embed"   rows of a [vocab, n] table by token number, times a factor; a share ``padded`` of the
            ``count`` numbers is -1 (a row of zeros); with ``train`` the table's gradient too
  "loss"    softmax cross entropy of [rows, n] hidden states against a [vocab, n] table without
            its logits: a row's loss and the logarithm of its sum; a share ``left_out`` of the
            rows has no target; ``pairs`` scores unit vectors against unit vectors (row i belongs
            to row i); with ``train`` the gradients of both, from weights of the rows that are
            equal or ``ragged``
  "orth"    a stack of ``count`` matrices [m, n] made nearly orthogonal by five steps of
            X <- a X + (b A + c A A) X with A = X X^T
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
WHOLE = {"i32": torch.int32, "i64": torch.int64}
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def _embed(name, count, vocab, n, tdtype, dtype, *, ids="i64", padded=0.0, train=False):
    c = dict(op="embed", count=count, vocab=vocab, n=n, tdtype=tdtype, dtype=dtype, ids=ids,
             padded=padded, train=train)
    return dict(c, name=name) if name else c


def _loss(name, rows, vocab, n, dtype, *, scale=1.0, pairs=False, left_out=0.0, ragged=False,
          train=False):
    c = dict(op="loss", rows=rows, vocab=vocab, n=n, dtype=dtype, scale=scale, pairs=pairs,
             left_out=left_out, ragged=ragged, train=train)
    return dict(c, name=name) if name else c


def _orth(name, count, m, n, dtype):
    c = dict(op="orth", count=count, m=m, n=n, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short text at ingest: launches and latency
        _embed("embed_one_text_24x768_f16", 24, 32768, 768, "f16", "f16"),
        # a large corpus batch embedded at the width of the 768-dimension index
        _embed("embed_corpus_262144x768_f16", 262144, 32768, 768, "f16", "f16"),
        # a training batch: a table kept in 32 bits, activations in 16, and some padding
        _embed("embed_train_65536x1024_f32_bf16", 65536, 50000, 1024, "f32", "bf16", padded=0.05,
               train=True),
        # a ragged token count, a width that is no multiple of a vector load, a small table
        _embed("embed_train_20001x515_f32", 20001, 2000, 515, "f32", "f32", ids="i32",
               train=True),
        # the likelihood of one token, and of one short text: the table is read once
        _loss("loss_one_token_32768x768_f16", 1, 32768, 768, "f16"),
        # pairs of near duplicates, every other document of the batch a negative
        _loss("loss_train_pairs_2048_768_f16", 2048, 2048, 768, "f16", scale=20.0, pairs=True,
              train=True),
        # the masked tokens of a training batch
        _loss("loss_train_8192x32768x768_bf16", 8192, 32768, 768, "bf16", left_out=0.1,
              train=True),
        # a large ragged batch over a large odd vocabulary, rows weighed by their documents
        _loss("loss_train_12007x100003x1024_bf16", 12007, 100003, 1024, "bf16", left_out=0.1,
              ragged=True, train=True),
        # 32-bit training of a small encoder: odd sizes everywhere
        _loss("loss_train_2001x7919x515_f32", 2001, 7919, 515, "f32", left_out=0.1, ragged=True,
              train=True),
        # one projection of a small encoder
        _orth("orth_one_256x256_f32", 1, 256, 256, "f32"),
        # the square projections of twelve layers
        _orth("orth_layers_36x768x768_bf16", 36, 768, 768, "bf16"),
        # wide projections in 32 bits
        _orth("orth_wide_8x1024x4096_f32", 8, 1024, 4096, "f32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_train", "score", "loss_train", "loss_train", "pairs",
                       "orth", "orth"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    widths = [64, 77, 256, 384, 512, 515, 768, 1000, 1024, 2048]
    if kind.startswith("embed"):
        n = rng.choice(widths)
        train = kind == "embed_train"
        count = min(_log(rng, 1, 262144), 2 ** 27 // n if not train else 2 ** 26 // n)
        vocab = min(_log(rng, 50, 150000), 2 ** 26 // n)
        return _embed(None, count, vocab, n, rng.choice([dtype, "f32"]), dtype,
                      ids=rng.choice(["i32", "i64"]), padded=rng.choice([0.0, 0.05]), train=train)
    if kind == "orth":
        # up to a quarter of the largest listed case's products
        m = _log(rng, 16, 2100)
        n = min(4096, max(16, int(m * rng.choice([0.25, 0.5, 1, 1, 1, 2, 4]) + rng.choice([0, 1]))))
        short, long_ = min(m, n), max(m, n)
        most = 2 ** 33 // (short * short * (2 * long_ + short))
        return _orth(None, max(1, min(_log(rng, 1, 48), most)), m, n, dtype)
    n = rng.choice(widths)
    if kind == "pairs":
        rows = _log(rng, 8, 4096)
        return _loss(None, rows, rows * rng.choice([1, 1, 2]), n, dtype,
                     scale=rng.choice([10.0, 20.0, 50.0]), pairs=True, train=True)
    train = kind == "loss_train"
    vocab = min(_log(rng, 50, 131072), 2 ** 27 // n)
    rows = max(1, min(_log(rng, 1, 8192), 2 ** 38 // (vocab * n)))
    return _loss(None, rows, vocab, n, dtype, left_out=rng.choice([0.0, 0.1]) if rows > 20 else 0.0,
                 ragged=rng.random() < 0.5, train=train)


def _bytes(dtype):
    return 4 if dtype == "f32" else 2


def work(case):
    c = case
    if c["op"] == "embed":
        live = round(c["count"] * (1 - c["padded"]))
        ids = c["count"] * (4 if c["ids"] == "i32" else 8)
        table = c["vocab"] * c["n"] * _bytes(c["tdtype"])
        grid = c["count"] * c["n"] * _bytes(c["dtype"])
        read = min(live * c["n"] * _bytes(c["tdtype"]), table)
        total = ids + read + grid
        if c["train"]:
            total += live * c["n"] * _bytes(c["dtype"]) + table
        return {"bytes": total, "flops": live * c["n"] * (2 if c["train"] else 1)}
    if c["op"] == "loss":
        size = _bytes(c["dtype"])
        read = (c["rows"] + c["vocab"]) * c["n"] * size + c["rows"] * 8
        product = 2 * c["rows"] * c["vocab"] * c["n"]
        if not c["train"]:
            return {"bytes": read + 8 * c["rows"], "flops": product}
        # both gradients written; the logits, and a product for each gradient
        return {"bytes": 2 * read + 20 * c["rows"], "flops": 3 * product}
    short, long_ = min(c["m"], c["n"]), max(c["m"], c["n"])
    # X X^T and A A are symmetric: half of each product is enough
    step = short * short * long_ + short ** 3 + 2 * short * short * long_
    return {"bytes": 2 * c["count"] * c["m"] * c["n"] * _bytes(c["dtype"]),
            "flops": STEPS * c["count"] * step}


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _words(count, vocab, g, dev):
    """Token numbers as text has them: the r-th most frequent one about 1 / (r + 3) of the time,
    frequent ones spread over the table."""
    u = torch.rand(count, generator=g, device=dev, dtype=torch.float64)
    rank = (3.0 * torch.exp(u * math.log((vocab + 3.0) / 3.0)) - 3.0).long().clamp_(0, vocab - 1)
    step = next(s for s in (7919, 6101, 4099, 2053, 1) if math.gcd(s, vocab) == 1)
    return (rank * step + 11) % vocab


def prepare(case, seed):
    c, dev = case, _device()
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 13)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=dev) * scale

    s = {"case": c}
    if c["op"] == "embed":
        ids = _words(c["count"], c["vocab"], g, dev)
        out = torch.rand(c["count"], generator=g, device=dev) < c["padded"]
        s["ids"] = torch.where(out, -1, ids).to(WHOLE[c["ids"]])
        s["table"] = normal(c["vocab"], c["n"], scale=c["n"] ** -0.5).to(DTYPES[c["tdtype"]])
        if c["train"]:
            s["dy"] = normal(c["count"], c["n"], scale=0.05).to(DTYPES[c["dtype"]])
        return s
    if c["op"] == "loss":
        dt, rows, vocab, n = DTYPES[c["dtype"]], c["rows"], c["vocab"], c["n"]
        if c["pairs"]:
            # half of the pairs are near, the others hardly alike
            table = torch.nn.functional.normalize(normal(vocab, n), dim=1)
            target = torch.arange(rows, device=dev)
            near = torch.rand(rows, 1, generator=g, device=dev)
            noise = torch.nn.functional.normalize(normal(rows, n), dim=1)
            h = torch.nn.functional.normalize(near * table[:rows] + (1 - near) * noise, dim=1)
        else:
            # normed hidden states that point, some more than others, at their word's row
            table = normal(vocab, n, scale=1.5 * n ** -0.5)
            target = _words(rows, vocab, g, dev)
            toward = 8.0 * torch.rand(rows, 1, generator=g, device=dev)
            h = normal(rows, n) + toward * table[target] / 2.25
        s["h"], s["table"] = h.to(dt), table.to(dt)
        out = torch.rand(rows, generator=g, device=dev) < c["left_out"]
        s["targets"] = torch.where(out, -100, target)
        if c["train"]:
            live = ~out
            weight = live.float()
            if c["ragged"]:
                weight = weight * (0.1 + torch.rand(rows, generator=g, device=dev))
            s["dloss"] = weight / live.sum().clamp(min=1)
        return s
    # momentum of a projection: a few strong directions over a decaying rest
    m, n, k = c["m"], c["n"], min(c["m"], c["n"], 32)
    strong = normal(c["count"], m, k) * torch.exp(-0.15 * torch.arange(k, device=dev))
    x = torch.bmm(strong, normal(c["count"], k, n)) * 0.05
    channel = torch.exp(0.7 * normal(c["count"], 1, n))
    s["g"] = ((x + 0.1 * normal(c["count"], m, n) * channel) * 1e-3).to(DTYPES[c["dtype"]])
    return s


def run(state):
    c = state["case"]
    if own:
        return _OWN[c["op"]](state, c)
    return _PLAIN[c["op"]](state, c)


def _embed_own(s, c):
    import paper_2608_03199_amd as ps
    scale = math.sqrt(c["n"])
    out = {"out": ps.embed_forward(s["ids"], s["table"], scale, dtype=DTYPES[c["dtype"]])}
    if c["train"]:
        out["dtable"] = ps.embed_backward(s["dy"], s["ids"], c["vocab"], scale,
                                          dtype=DTYPES[c["tdtype"]])
    return out


def _loss_own(s, c):
    import paper_2608_03199_amd as ps
    loss, lse = ps.linear_cross_entropy_forward(s["h"], s["table"], s["targets"], c["scale"])
    out = {"loss": loss, "lse": lse}
    if c["train"]:
        out["dh"], out["dtable"] = ps.linear_cross_entropy_backward(
            s["dloss"], s["h"], s["table"], s["targets"], lse, c["scale"])
    return out


def _orth_own(s, c):
    import paper_2608_03199_amd as ps
    return {"x": ps.orthogonalize(s["g"], STEPS, COEFFICIENTS, EPS)}


_OWN = {"embed": _embed_own, "loss": _loss_own, "orth": _orth_own}


def _embed_plain(s, c):
    live, scale = s["ids"] >= 0, math.sqrt(c["n"])
    rows = s["table"][torch.where(live, s["ids"], 0)].float() * scale
    out = {"out": torch.where(live[:, None], rows, 0.0).to(DTYPES[c["dtype"]])}
    if c["train"]:
        # the rows that are left out are added to one row more
        at = torch.where(live, s["ids"], c["vocab"])
        grad = torch.zeros(c["vocab"] + 1, c["n"], device=at.device)
        grad.index_add_(0, at, s["dy"].float())
        out["dtable"] = (grad[:-1] * scale).to(DTYPES[c["tdtype"]])
    return out


def _loss_plain(s, c):
    h, table = s["h"].float(), s["table"].float()
    live = s["targets"] >= 0
    target = torch.where(live, s["targets"], 0)
    logits = torch.matmul(h, table.t()) * c["scale"]
    top = logits.amax(1, keepdim=True)
    lse = top + torch.exp(logits - top).sum(1, keepdim=True).log()
    loss = (lse - logits.gather(1, target[:, None]))[:, 0]
    out = {"loss": torch.where(live, loss, 0.0), "lse": lse[:, 0]}
    if c["train"]:
        d = logits.sub_(lse).exp_()
        d[torch.arange(d.shape[0], device=d.device), target] -= 1
        d *= (s["dloss"] * live * c["scale"])[:, None]
        out["dh"] = torch.matmul(d, table).to(s["h"].dtype)
        out["dtable"] = torch.matmul(d.t(), h).to(s["table"].dtype)
    return out


def _orth_plain(s, c):
    a, b, d = COEFFICIENTS
    x = s["g"].float()
    tall = c["m"] > c["n"]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + d * torch.bmm(gram, gram), x)
    if tall:
        x = x.transpose(1, 2)
    return {"x": x.to(s["g"].dtype).contiguous()}


_PLAIN = {"embed": _embed_plain, "loss": _loss_plain, "orth": _orth_plain}


def exact(case, seed):
    return _EXACT[case["op"]](prepare(case, seed), case)


def _embed_exact(s, c):
    scale, n = math.sqrt(c["n"]), c["n"]
    out = torch.zeros(c["count"], n, dtype=torch.float64, device=s["ids"].device)
    live = torch.nonzero(s["ids"] >= 0)[:, 0]
    ids = s["ids"].long()[live]
    out[live] = s["table"].double().index_select(0, ids) * scale
    got = {"out": out}
    if c["train"]:
        # tokens in the order of their numbers, sums of runs as differences of running sums
        order = torch.argsort(ids, stable=True)
        count = torch.bincount(ids, minlength=c["vocab"])
        end = count.cumsum(0)
        grad = torch.zeros(c["vocab"], n, dtype=torch.float64, device=ids.device)
        for a in range(0, n, 128):  # pieces of the columns, for memory
            run_ = s["dy"][:, a:a + 128][live[order]].double().cumsum(0)
            run_ = torch.cat([torch.zeros_like(run_[:1]), run_])
            grad[:, a:a + 128] = (run_[end] - run_[end - count]) * scale
        got["dtable"] = grad
    return got


def _loss_exact(s, c):
    if c["rows"] * c["vocab"] * c["n"] > 2 ** 41:
        return None
    h, w, train = s["h"].double(), s["table"].double(), c["train"]
    got = {k: torch.zeros(c["rows"], dtype=torch.float64, device=h.device) for k in ("loss", "lse")}
    if train:
        got.update(dh=torch.zeros_like(h), dtable=torch.zeros_like(w))
    per = max(1, 2 ** 28 // c["vocab"])
    for at in torch.arange(c["rows"], device=h.device).split(per):  # pieces, for memory
        logits = c["scale"] * (h[at] @ w.t())
        got["lse"][at] = torch.logsumexp(logits, 1)
        some = s["targets"][at] >= 0
        at, logits = at[some], logits[some]
        here = (torch.arange(len(at), device=h.device), s["targets"][at])
        got["loss"][at] = got["lse"][at] - logits[here]
        if train:
            p = torch.softmax(logits, 1)
            p[here] -= 1.0
            p *= s["dloss"][at].double()[:, None] * c["scale"]
            got["dh"][at] = p @ w
            got["dtable"] += p.t() @ h[at]
    return got


def _orth_exact(s, c):
    a, b, d = COEFFICIENTS
    x = s["g"].double()
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    eye = torch.eye(min(c["m"], c["n"]), dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        if c["m"] > c["n"]:
            gram = x.mT @ x
            x = x @ (a * eye + gram @ (b * eye + d * gram))
        else:
            gram = x @ x.mT
            x = (a * eye + gram @ (b * eye + d * gram)) @ x
    return {"x": x}


_EXACT = {"embed": _embed_exact, "loss": _loss_exact, "orth": _orth_exact}
