"""The operators together in the example's training step: the contrastive loss's gradients against
torch's, and a run with orthogonalised momentum."""
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


def test_contrastive_step_gradients_against_torch(example):
    """Gradients of every parameter through the library's loss, and through torch's products and
    cross entropy behind the same fp32 encoder.  Both are fp32 from the embeddings on, unit vectors
    of 256 values whose scores are scaled by 20 and summed over 16: the two losses' gradients
    differ by some 256 20 2^-24 of the largest, and what the encoder makes of that is linear."""
    ps = example.ps
    torch.manual_seed(0)
    model = example.Encoder(torch.float32)
    docs = example.make_documents(32, torch.Generator().manual_seed(3))
    batch = example.Batch(docs, torch.float32)
    target = torch.arange(16, device="cuda")
    grads = []
    for own in (True, False):
        model.zero_grad()
        e = model(batch)
        if own:
            loss = ps.linear_cross_entropy(e[0::2], e[1::2], target, 20.0).mean()
        else:
            score = (e[0::2, None] * e[None, 1::2]).sum(2) * 20.0
            loss = (torch.logsumexp(score, 1) - score[target, target]).mean()
        loss.backward()
        grads.append({n: p.grad.double().clone() for n, p in model.named_parameters()})
    for name, want in grads[1].items():
        bound = 16 * 256 * 20 * 2.0 ** -24 * float(want.abs().max())
        assert float((grads[0][name] - want).abs().max()) <= bound, name


def test_orthogonal_update(example):
    """A step moves each matrix along its orthogonalised momentum, by the rate."""
    from training_reference import near, orthogonalize_bound
    torch.manual_seed(1)
    p = [torch.nn.Parameter(torch.randn(*s, device="cuda")) for s in ((40, 60), (60, 40), (40, 60))]
    opt = example.Orthogonal(p, lr=0.5, beta=0.5)
    momentum = [torch.zeros_like(x).cpu() for x in p]
    for _ in range(2):
        before = [x.detach().clone() for x in p]
        for i, x in enumerate(p):
            x.grad = torch.randn_like(x)
            momentum[i] = 0.5 * momentum[i] + x.grad.cpu()
        opt.step()
        for i, x in enumerate(p):
            rate = 0.5 * max(1.0, x.shape[1] / x.shape[0]) ** 0.5
            val, bound = orthogonalize_bound(momentum[i], 5, (3.4445, -4.7750, 2.0315), 1e-7)
            # the difference of two fp32 weights of about 1 to 4 is good to 2^-22
            moved = (before[i] - x.detach()).double().cpu() / rate
            near("step", moved, val, bound + 2.0 ** -22 * 4 / rate * 40 ** 0.5)


def test_training_with_orthogonal_momentum_runs(example):
    losses, found, _ = example.main(["--docs", "64", "--steps", "3", "--pairs", "16",
                                     "--orthogonal"])
    assert len(losses) == 3 and all(x == x for x in losses)
