"""The operators around the encoder's blocks in 64 bits on the CPU, with bounds on how far a
computation in a given type may be from them.

Bounds follow the operations: products and sums in fp32 (unit roundoff E), values rounded to a
type (unit roundoff u) where the operators round them."""
import torch

from encoder_reference import E, TINY, UNIT


def embed(ids, table, scale, dtype, dy=None, into=None):
    """({name: value}, {name: bound}) of the lookup, and of the table's gradient with dy."""
    vocab, n = table.shape
    flat = ids.reshape(-1).long()
    live = (flat >= 0) & (flat < vocab)
    rows = torch.where(live[:, None], table.double()[flat.clamp(0, vocab - 1)] * scale, 0.0)
    val = {"out": rows.reshape(ids.shape + (n,))}
    # the factor itself is fp32: E more
    tol = {"out": (UNIT[dtype] + 2 * E) * val["out"].abs() + TINY[dtype]}
    if dy is None:
        return val, tol
    d = dy.double().reshape(-1, n)[live]
    at = flat[live]
    total = torch.zeros(vocab, n, dtype=torch.float64).index_add_(0, at, d) * scale
    size = torch.zeros(vocab, n, dtype=torch.float64).index_add_(0, at, d.abs()) * abs(scale)
    if into is not None:
        total, size = total + into.double(), size + into.double().abs()
    # a value takes part in at most this many additions: 32 in a piece of each kind, and those
    # at the ends of the row's pieces (62 of each kind); two roundings of the factor, one of into
    kinds, span = 0, 32
    while span <= flat.numel():
        kinds, span = kinds + 1, span * 32
    steps = min(int(torch.bincount(at, minlength=1).max()) if len(at) else 0,
                32 * kinds + 62 * (kinds + 1)) + 3
    out = table.dtype if into is None else into.dtype
    val["dtable"] = total
    tol["dtable"] = UNIT[out] * total.abs() + (1 + UNIT[out]) * steps * E * size + TINY[out]
    return val, tol


def cross_entropy(h, table, targets, scale, dloss=None):
    """({name: value}, {name: bound}) of loss and lse, and of dh and dtable with dloss."""
    dt, n, vocab = h.dtype, h.shape[1], table.shape[0]
    u, c = UNIT[dt], float(torch.tensor(scale, dtype=torch.float32))
    x, w = h.double(), table.double()
    live = (targets >= 0) & (targets < vocab)
    at = targets.long().clamp(0, vocab - 1)
    s = c * (x @ w.T)
    # a logit: n products of 16-bit values, exact, or 6 n of 32-bit values' parts, added in fp32
    # (2 E each: the matrix units need not round to nearest); the parts left out are below 8 E
    terms = (6 * n + 16) * 2 * E if dt is torch.float32 else (n + 16) * 2 * E
    ds = c * (x.abs() @ w.abs().T) * (terms + 8 * E) + 4 * E * s.abs()
    lse = torch.logsumexp(s, 1)
    # exponentials and the logarithm to 2^-21, sums of up to vocab of them
    many = (min(vocab, 300) + vocab / 256 + 16) * E
    d_lse = ds.max(1).values + 2.0 ** -20 + many + 4 * E * (lse.abs() + s.abs().max(1).values)
    own = s.gather(1, at[:, None])[:, 0]
    loss = torch.where(live, lse - own, 0.0)
    val = {"lse": lse, "loss": loss}
    tol = {"lse": d_lse, "loss": (d_lse + ds.gather(1, at[:, None])[:, 0] + 4 * E * own.abs()) * live}
    if dloss is None:
        return val, tol
    weight = torch.where(live, dloss.double(), 0.0)
    p = torch.exp(s - lse[:, None])
    one = torch.zeros_like(p)
    one[torch.arange(len(at)), at] = 1.0
    g = (p - one) * weight[:, None]
    d_p = p * (ds + d_lse[:, None] + 2.0 ** -20 + 4 * E * (s.abs() + lse.abs()[:, None]))
    # rounded to the inputs' type, over the row's factor (which cancels)
    d_g = (1 + u) * d_p * weight.abs()[:, None] + (u + 8 * E) * g.abs()
    # an exponential below fp32's normal range (2^-126) may be zero, and so may g, or a part of it
    # that a matrix unit reads, below that of its type
    d_g = d_g + 2.0 ** -126 * (weight.abs()[:, None] + 3)
    if dt is torch.float16:
        # scaled by 2^14, over a factor of at most dloss: a step of 2^-24 below the normal range
        d_g = d_g + 2.0 ** -39 * weight.abs()[:, None]

    def product(a, d_a, b, k, again=0.0):
        total = a @ b
        size, far = a.abs() @ b.abs(), (d_a + again * (a.abs() + d_a)) @ b.abs()
        parts = 6 * k if dt is torch.float32 else k
        e = c * (far + ((parts + 16) * 2 + 16) * E * (size + far))
        return c * total, e + u * (c * total.abs() + e) + TINY[dt]

    val["dh"], tol["dh"] = product(g, d_g, w, vocab)
    held = torch.where(weight[:, None] != 0, x, 0.0)
    # h is rounded once more, with its row's factor
    val["dtable"], tol["dtable"] = product(g.T, d_g.T, held, len(at), u + 4 * E)
    if dt is torch.float16:
        # rows of far smaller factors may fall below the type's normal range
        top = weight.abs().max() if len(at) else 0.0
        tol["dtable"] = tol["dtable"] + c * top * 2.0 ** -23 * (g != 0).sum(0)[:, None]
    return val, tol


def near(name, got, want, bound):
    """Whether the error's norm is at most ``bound`` times the value's."""
    d = float((got.detach().double().cpu() - want).norm())
    assert d <= bound * float(want.norm()), f"{name}: off by {d / float(want.norm()):.3g}"


def orthogonalize(g, steps, coefficients, eps, dtype=torch.float64):
    """The iteration in ``dtype``, on matrices as they lie."""
    a, b, c = coefficients
    x = g.to(dtype)
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        gram = x @ x.mT if x.shape[-2] <= x.shape[-1] else x.mT @ x
        poly = b * gram + c * gram @ gram
        x = a * x + (poly @ x if x.shape[-2] <= x.shape[-1] else x @ poly)
    return x


def orthogonalize_bound(g, steps, coefficients, eps):
    """(value, bound of the error's norm over the value's).  Rounding errors grow with what is
    weak in g, and nothing simpler than the iteration itself says by how much: the bound is four
    times what fp32 arithmetic gets (values of 24 bits in two parts, three of their four products,
    sums in fp32), and a rounding of the result."""
    val = orthogonalize(g, steps, coefficients, eps)
    single = orthogonalize(g, steps, coefficients, eps, torch.float32).double()
    off = float((single - val).norm() / val.norm())
    return val, 4 * off + 8 * E + (UNIT[g.dtype] if g.dtype is not torch.float32 else 0.0)
