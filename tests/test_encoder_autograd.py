"""CPU-side checks of what torch's differentiation hands to the layer norm's backward kernel: the
kernels are replaced with plain code that records its arguments."""
import os

import pytest
import torch


@pytest.fixture()
def enc(monkeypatch):
    import paper_2608_03199_amd as ps
    if not os.path.exists(ps.LIB_PATH):
        from paper_2608_03199_amd import build
        build.build()
    from paper_2608_03199_amd import encoder
    calls = []

    def forward(x, weight, bias=None, eps=1e-5, residual=None, stream=None):
        h = x if residual is None else x + residual
        mean = h.mean(-1)
        rstd = 1 / torch.sqrt(h.var(-1, correction=0) + eps)
        y = (h - mean[..., None]) * rstd[..., None] * weight
        return (y if bias is None else y + bias), h, mean, rstd

    def backward(dy, h, weight, mean, rstd, dh=None, weight_grad=True, bias_grad=True,
                 stream=None):
        calls.append(dh)
        u = (h - mean[..., None]) * rstd[..., None]
        g = dy * weight
        dx = rstd[..., None] * (g - g.mean(-1, keepdim=True) - u * (g * u).mean(-1, keepdim=True))
        axes = tuple(range(h.dim() - 1))
        return (dx if dh is None else dx + dh, (dy * u).sum(axes) if weight_grad else None,
                dy.sum(axes) if bias_grad else None)

    monkeypatch.setattr(encoder, "layer_norm_forward", forward)
    monkeypatch.setattr(encoder, "layer_norm_backward", backward)
    encoder.calls = calls
    yield encoder
    del encoder.calls


@pytest.mark.parametrize("use", ["y", "h", "both", "plain"])
@pytest.mark.parametrize("bias", [False, True])
def test_norm_backward_reads_only_gradients_that_are_there(enc, use, bias):
    g = torch.Generator().manual_seed(1)
    x, r = (torch.randn(3, 4, 8, generator=g, dtype=torch.float64).requires_grad_() for _ in "xr")
    w = torch.randn(8, generator=g, dtype=torch.float64).requires_grad_()
    b = torch.randn(8, generator=g, dtype=torch.float64).requires_grad_() if bias else None
    dy, dh = (torch.randn(3, 4, 8, generator=g, dtype=torch.float64) for _ in "yh")
    leaves = [t for t in (x, w, b) + (() if use == "plain" else (r,)) if t is not None]

    def total(norm):
        if use == "plain":
            return (norm(None) * dy).sum()
        y, h = norm(r)
        return ((y * dy).sum() if use != "h" else 0) + ((h * dh).sum() if use != "y" else 0)

    got = torch.autograd.grad(total(lambda r: enc.layer_norm(x, w, b, 1e-5, r)), leaves)

    def plain(r):
        h = x if r is None else x + r
        y = torch.nn.functional.layer_norm(h, (8,), w, b, 1e-5)
        return y if r is None else (y, h)

    want = torch.autograd.grad(total(plain), leaves, allow_unused=True)
    for a, e in zip(got, want):
        assert torch.allclose(a, torch.zeros_like(a) if e is None else e, rtol=1e-12, atol=1e-12)
    # no zeros in the place of a gradient that is not there, and no kernel where there is none
    assert [c is None for c in enc.calls] == {"y": [True], "h": [], "both": [False],
                                              "plain": [True]}[use]
