"""CPU-side checks of the operators around the encoder's blocks: argument errors before any HIP
call, limits, workspaces."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2608_03199_amd as ps
    if not os.path.exists(ps.LIB_PATH):
        from paper_2608_03199_amd import build
        build.build()
    from paper_2608_03199_amd import training
    return training._library()


P, NONE = ctypes.c_void_p(0x1000), None


def test_embed_argument_errors_without_a_gpu(lib):
    def forward(ids=P, size=8, count=4, table=P, stride=8, tdt=0, vocab=5, n=8, out=P, dt=0):
        return lib.sieve_embed_forward(ids, size, count, table, stride, tdt, vocab, n, 1.0, out,
                                       dt, NONE)

    assert forward(dt=3) == -1 and b"dtype" in lib.sieve_last_error()
    assert forward(tdt=1, dt=2) == -1 and b"tdtype" in lib.sieve_last_error()
    assert forward(tdt=1, dt=0) == -1
    assert forward(size=2) == -1 and b"id_bytes" in lib.sieve_last_error()
    assert forward(count=-1) == -1 and forward(vocab=0) == -1 and forward(n=0) == -1
    assert forward(n=65537, stride=65537) == -4
    assert forward(count=1 << 31) == -4 and forward(vocab=(1 << 31) - 1) == -4
    assert forward(ids=NONE) == -1 and forward(table=NONE) == -1 and forward(out=NONE) == -1
    assert forward(stride=7) == -1 and b"stride" in lib.sieve_last_error()
    assert forward(count=0, ids=NONE, out=NONE) == 0

    def backward(dy=P, stride=8, dt=0, ids=P, size=8, count=4, vocab=5, n=8, acc=0, out=P, tdt=0,
                 ws=P, bytes=1 << 30):
        return lib.sieve_embed_backward(dy, stride, dt, ids, size, count, vocab, n, 1.0, acc, out,
                                        tdt, ws, bytes, NONE)

    assert backward(acc=2) == -1 and b"accumulate" in lib.sieve_last_error()
    assert backward(out=NONE) == -1 and backward(dy=NONE) == -1 and backward(ids=NONE) == -1
    assert backward(stride=7) == -1
    assert backward(ws=NONE) == -1 and b"workspace" in lib.sieve_last_error()
    assert backward(ws=ctypes.c_void_p(0x1008)) == -1 and backward(bytes=100) == -1
    assert backward(count=0, acc=1, dy=NONE, ids=NONE, ws=NONE, bytes=0) == 0
    assert lib.sieve_embed_workspace(0, 5, 8) == 0
    assert lib.sieve_embed_workspace(4, 0, 8) == -1 and lib.sieve_embed_workspace(4, 5, 0) == -1
    # two pairs of whole numbers a token, and a 1/31 of the batch's rows in fp32
    assert 16 * 65536 < lib.sieve_embed_workspace(65536, 50000, 1024) < \
        16 * 65536 + 65536 * 1024 * 4 // 31 + (1 << 20)
    assert lib.sieve_embed_workspace((1 << 31) - 1, (1 << 31) - 2, 65536) > 0


def test_loss_argument_errors_without_a_gpu(lib):
    def forward(h=P, hs=8, table=P, ts=8, dt=0, rows=4, vocab=5, n=8, targets=P, size=8, scale=1.0,
                lse=P, ws=P, bytes=1 << 40):
        return lib.sieve_loss_forward(h, hs, table, ts, dt, rows, vocab, n, targets, size, scale, P,
                                      lse, ws, bytes, NONE)

    assert forward(dt=3) == -1 and b"dtype" in lib.sieve_last_error()
    assert forward(rows=-1) == -1 and forward(vocab=0) == -1 and forward(n=0) == -1
    assert forward(n=65537, hs=65537, ts=65537) == -4
    assert forward(rows=(1 << 24) + 1) == -4 and forward(vocab=(1 << 24) + 1) == -4
    assert forward(h=NONE) == -1 and forward(table=NONE) == -1 and forward(targets=NONE) == -1
    assert forward(lse=NONE) == -1
    assert forward(size=2) == -1 and b"target_bytes" in lib.sieve_last_error()
    assert forward(hs=7) == -1 and forward(ts=7) == -1
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert forward(scale=scale) == -1 and b"scale" in lib.sieve_last_error()
    assert forward(ws=NONE) == -1 and forward(ws=ctypes.c_void_p(0x1008)) == -1
    assert forward(bytes=16) == -1 and b"workspace" in lib.sieve_last_error()
    assert forward(rows=0, h=NONE, targets=NONE, ws=NONE) == 0

    def backward(dloss=P, h=P, table=P, rows=4, lse=P, scale=1.0, dh=P, dtable=P, ws=P,
                 bytes=1 << 40, dt=0, vocab=5):
        return lib.sieve_loss_backward(dloss, h, 8, table, 8, dt, rows, vocab, 8, P, 8, lse, scale,
                                       dh, dtable, ws, bytes, NONE)

    assert backward(dt=-1) == -1 and backward(vocab=0) == -1
    assert backward(dloss=NONE) == -1 and backward(lse=NONE) == -1 and backward(h=NONE) == -1
    assert backward(scale=0.0) == -1 and backward(ws=NONE) == -1 and backward(bytes=16) == -1
    assert backward(dh=NONE, dtable=NONE) == 0
    assert backward(rows=0, dtable=NONE, ws=NONE) == 0
    assert lib.sieve_loss_workspace(4, 5, 8, 0, 2) == -1
    assert lib.sieve_loss_workspace(4, 5, 8, 7, 0) == -1
    assert lib.sieve_loss_workspace(0, 5, 8, 0, 1) == 0
    # no logits: a large vocabulary takes no more than some pieces of its gradients
    assert lib.sieve_loss_workspace(8192, 1 << 20, 768, 2, 0) < 8192 * (1 << 20) * 2 // 16
    assert lib.sieve_loss_workspace(8192, 1 << 20, 768, 2, 1) < 8192 * (1 << 20) * 2 // 16


def test_orthogonalize_argument_errors_without_a_gpu(lib):
    def call(g=P, bs=64, rs=8, dt=0, batch=1, m=8, n=8, steps=5, c=(3.4445, -4.775, 2.0315),
             eps=1e-7, x=P, ws=P, bytes=1 << 40):
        three = None if c is None else (ctypes.c_float * 3)(*c)
        return lib.sieve_orthogonalize(g, bs, rs, dt, batch, m, n, steps, three, eps, x, ws, bytes,
                                       NONE)

    inf, nan = float("inf"), float("nan")
    assert call(dt=3) == -1 and call(batch=-1) == -1 and call(m=0) == -1 and call(n=0) == -1
    assert call(m=65537) == -4 and call(n=65537, rs=65537) == -4
    assert call(steps=-1) == -1 and call(steps=1001) == -4
    assert call(eps=-1.0) == -1 and call(eps=nan) == -1 and call(eps=inf) == -1
    assert call(c=None) == -1 and call(c=(nan, 0, 0)) == -1 and call(c=(1, inf, 0)) == -1
    assert call(g=NONE) == -1 and call(x=NONE) == -1 and call(rs=7) == -1 and call(bs=-1) == -1
    assert call(ws=NONE) == -1 and call(ws=ctypes.c_void_p(0x1008)) == -1 and call(bytes=8) == -1
    assert call(batch=0, g=NONE, x=NONE, ws=NONE) == 0
    # coefficients with which singular values leave the range: checked for the steps asked for
    assert call(batch=0, steps=7, c=(1.2, 0, 0)) == 0 and call(batch=0, steps=8, c=(1.2, 0, 0)) == -4
    assert call(batch=0, c=(16, -30, 14.5)) == -4 and b"singular" in lib.sieve_last_error()
    assert call(batch=0, steps=1, c=(3.8, 0, 0)) == 0 and call(batch=0, steps=1, c=(4, 0, 0)) == -4
    assert call(batch=0, steps=1000, c=(1.875, -1.25, 0.375)) == 0
    assert call(batch=0, steps=1000, c=(3.4445, -4.775, 2.0315)) == 0
    # a maximum inside [0, 1]: 8 x - 8 x^3 reaches 3.08 at 0.577 and is 0 at both ends
    assert call(batch=0, steps=1, c=(8, -8, 0)) == 0 and call(batch=0, steps=1, c=(11, -11, 0)) == -4
    assert lib.sieve_orthogonalize_workspace(0, 8, 8) == 0
    assert lib.sieve_orthogonalize_workspace(1, 0, 8) == -1
    # X twice, and three products, each in two parts of 2 bytes
    assert lib.sieve_orthogonalize_workspace(2, 64, 128) == 2 * 4 * (2 * 64 * 128 + 3 * 64 * 64) + 1024
