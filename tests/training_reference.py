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
