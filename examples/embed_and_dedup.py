"""A text encoder trained on near-duplicate pairs, its embeddings, and their self-join.

The library's operators as they are used together: documents of ragged lengths are packed, an
encoder block runs layer norm and attention with a learned relative position bias over the
packed batch, one query per document pools its tokens, a contrastive loss trains all of it on
pairs of near duplicates, and the embedded corpus is loaded into an index and joined with itself
at a threshold.  The matrix products around the operators are torch's.

    python examples/embed_and_dedup.py [--docs 2000] [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_03199_amd as ps  # noqa: E402

VOCAB, HEADS, HEAD_DIM, LAYERS, BUCKETS, DISTANCE = 2000, 4, 64, 2, 32, 128
WIDTH = HEADS * HEAD_DIM


class Batch:
    """Packed documents: tokens one after another, offsets, and the two attention plans that
    every layer and the backward pass share (tokens among each other; a pooling query each)."""

    def __init__(self, docs, dtype):
        lens = torch.tensor([len(d) for d in docs])
        self.offsets = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
        self.tokens = torch.cat(docs).cuda()
        shape = dict(heads=HEADS, head_dim=HEAD_DIM, dtype=dtype)
        self.plan = ps.AttentionPlan(self.offsets, num_buckets=BUCKETS, max_distance=DISTANCE,
                                     **shape)
        self.pool = ps.AttentionPlan(torch.arange(len(docs) + 1), self.offsets, **shape)
        self.size = len(docs)


class Encoder(torch.nn.Module):
    def __init__(self, dtype=torch.bfloat16):
        super().__init__()
        self.dtype = dtype

        def weight(*shape, scale=None):
            scale = shape[0] ** -0.5 if scale is None else scale
            return torch.nn.Parameter(torch.randn(*shape, device="cuda") * scale)

        self.embed = weight(VOCAB, WIDTH, scale=1.0)
        self.bias = weight(BUCKETS, HEADS, scale=0.1)
        self.query = weight(HEADS, HEAD_DIM, scale=0.1)
        self.layers = torch.nn.ModuleList()
        for _ in range(LAYERS):
            self.layers.append(torch.nn.ParameterDict(dict(
                qkv=weight(WIDTH, 3 * WIDTH), out=weight(WIDTH, WIDTH),
                up=weight(WIDTH, 2 * WIDTH), down=weight(2 * WIDTH, WIDTH),
                norm1=torch.nn.Parameter(torch.ones(WIDTH, device="cuda")),
                bias1=torch.nn.Parameter(torch.zeros(WIDTH, device="cuda")),
                norm2=torch.nn.Parameter(torch.ones(WIDTH, device="cuda")),
                bias2=torch.nn.Parameter(torch.zeros(WIDTH, device="cuda")))))

    def forward(self, batch):
        dt = self.dtype
        h = self.embed.to(dt)[batch.tokens]
        bias = self.bias.to(dt)  # one table for all layers
        branch = torch.zeros_like(h)
        for p in self.layers:
            # the residual sum and the norm of it in one pass
            x, h = ps.layer_norm(branch, p["norm1"], p["bias1"], residual=h)
            q, k, v = (x @ p["qkv"].to(dt)).view(-1, 3, HEADS, HEAD_DIM).unbind(1)
            a = ps.attention(q, k, v, batch.plan, bias=bias)
            x, h = ps.layer_norm(a.reshape(-1, WIDTH) @ p["out"].to(dt), p["norm2"], p["bias2"],
                                 residual=h)
            branch = torch.relu(x @ p["up"].to(dt)) @ p["down"].to(dt)
        tokens = (h + branch).view(-1, HEADS, HEAD_DIM)
        query = self.query.to(dt).expand(batch.size, HEADS, HEAD_DIM)
        pooled = ps.attention(query, tokens, tokens, batch.pool).reshape(-1, WIDTH).float()
        return torch.nn.functional.normalize(pooled, dim=1)


def make_documents(count, generator):
    """Documents of 8..200 tokens; every second one repeats the one before it with a tenth of
    its tokens changed."""
    docs = []
    for i in range(count):
        if i % 2:
            d = docs[-1].clone()
            change = torch.rand(len(d), generator=generator) < 0.1
            d[change] = torch.randint(VOCAB, (int(change.sum()),), generator=generator)
        else:
            n = int(torch.randint(8, 201, (1,), generator=generator))
            d = torch.randint(VOCAB, (n,), generator=generator)
        docs.append(d)
    return docs


def train(model, steps, pairs, generator, say=print):
    opt = torch.optim.Adam(model.parameters(), lr=2e-3)
    losses = []
    for step in range(steps):
        batch = Batch(make_documents(2 * pairs, generator), model.dtype)
        e = model(batch)
        score = e[0::2] @ e[1::2].T / 0.05
        target = torch.arange(pairs, device="cuda")
        loss = torch.nn.functional.cross_entropy(score, target)
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        if step % 20 == 0 or step == steps - 1:
            say(f"step {step}: loss {losses[-1]:.4f}")
    return losses


def embed(model, docs, size=512):
    with torch.no_grad():
        return torch.cat([model(Batch(docs[i:i + size], model.dtype))
                          for i in range(0, len(docs), size)])


def self_join(vectors, tau, nlist=16):
    """Neighbours at or above tau of every row, by the index: (ids, scores) as search returns."""
    n = vectors.shape[0]
    x = vectors.half()
    centroids = x[torch.randperm(n, generator=torch.Generator().manual_seed(0))[:nlist].cuda()]
    for _ in range(3):
        near = (x.float() @ centroids.float().T).argmax(1)
        total = torch.zeros(nlist, x.shape[1], device="cuda").index_add_(0, near, x.float())
        centroids = torch.where((total != 0).any(1, keepdim=True),
                                torch.nn.functional.normalize(total, dim=1),
                                centroids.float()).half()
    near = (x.float() @ centroids.float().T).argmax(1)
    order = torch.argsort(near, stable=True)
    offsets = torch.zeros(nlist + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.bincount(near, minlength=nlist).cumsum(0)
    ids = torch.arange(n, device="cuda")
    index = ps.Index(x[order].contiguous(), offsets, ids[order].contiguous(), centroids)
    try:
        found, scores, _ = index.search(x, ids, 10, tau, 8, nlist)
    finally:
        index.close()
    return found, scores


def main(argv=None):
    args = argparse.ArgumentParser()
    args.add_argument("--docs", type=int, default=2000)
    args.add_argument("--steps", type=int, default=60)
    args.add_argument("--pairs", type=int, default=128)
    args.add_argument("--tau", type=float, default=0.8)
    args = args.parse_args(argv)
    torch.manual_seed(0)
    g = torch.Generator().manual_seed(1)
    model = Encoder()
    losses = train(model, args.steps, args.pairs, g)
    docs = make_documents(args.docs // 2 * 2, g)
    found, _ = self_join(embed(model, docs), args.tau)
    partner = torch.arange(len(docs), device="cuda") ^ 1
    hit = (found == partner[:, None]).any(1)
    extra = ((found >= 0) & (found != partner[:, None])).sum()
    print(f"planted near duplicates found at {args.tau}: {int(hit.sum())} of {len(docs)}, "
          f"other neighbours: {int(extra)}")
    return losses, float(hit.float().mean()), int(extra)


if __name__ == "__main__":
    main()
