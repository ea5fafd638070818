"""The operators together: the example trains an encoder, embeds a corpus and joins it."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    spec = importlib.util.spec_from_file_location(
        "embed_and_dedup", os.path.join(ROOT, "examples", "embed_and_dedup.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_training_finds_the_planted_pairs(example):
    losses, found, _ = example.main(["--docs", "600", "--steps", "30", "--pairs", "64"])
    assert losses[-1] < 0.5 * losses[0]
    assert found > 0.9


def test_encoder_gradients_against_torch(example):
    """One step's gradients of every parameter in fp32 against the same encoder written with
    torch's own differentiation in 64 bits.  The loss sums each document's embedding with
    random weights, so the bound is relative to the largest entry of a parameter's gradient:
    fp32 through some 20 operations of at most 512 terms each."""
    torch.manual_seed(0)
    model = example.Encoder(torch.float32)
    g = torch.Generator().manual_seed(5)
    docs = example.make_documents(12, g)
    batch = example.Batch(docs, torch.float32)
    way = torch.randn(12, example.WIDTH, generator=g)
    (model(batch) * way.cuda()).sum().backward()

    params = {n: p.detach().double().cpu().requires_grad_() for n, p in model.named_parameters()}
    heads, dim, width = example.HEADS, example.HEAD_DIM, example.WIDTH

    def norm(x, w, b):
        c = x - x.mean(1, keepdim=True)
        return c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-5) * w + b

    from encoder_reference import bucket
    out = []
    for doc in docs:
        n = len(doc)
        rel = [[bucket(j - i, example.BUCKETS, example.DISTANCE, False) for j in range(n)]
               for i in range(n)]
        bias = params["bias"][torch.tensor(rel)].permute(2, 0, 1)
        h = params["embed"][doc]
        branch = torch.zeros_like(h)
        for layer in range(example.LAYERS):
            p = {k: params[f"layers.{layer}.{k}"] for k in ("qkv", "out", "up", "down", "norm1",
                                                            "bias1", "norm2", "bias2")}
            h = h + branch
            q, k, v = (norm(h, p["norm1"], p["bias1"]) @ p["qkv"]).view(n, 3, heads, dim) \
                .permute(1, 2, 0, 3)
            a = torch.softmax(q @ k.transpose(1, 2) / dim ** 0.5 + bias, 2) @ v
            h = h + a.transpose(0, 1).reshape(n, width) @ p["out"]
            branch = torch.relu(norm(h, p["norm2"], p["bias2"]) @ p["up"]) @ p["down"]
        t = (h + branch).view(n, heads, dim).transpose(0, 1)
        pool = torch.softmax(params["query"][:, None] @ t.transpose(1, 2) / dim ** 0.5, 2) @ t
        out.append(torch.nn.functional.normalize(pool.reshape(-1), dim=0))
    (torch.stack(out) * way.double()).sum().backward()
    for name, p in model.named_parameters():
        want = params[name].grad
        got = p.grad.double().cpu()
        assert float((got - want).abs().max()) <= 20 * 512 * 2.0 ** -24 * float(want.abs().max()), name
