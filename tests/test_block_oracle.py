"""Pins of the 64-bit definitions of dropout and layer norm, and what the C entry points refuse (argument checks come
before any CUDA call, so they run without a GPU)."""
import ctypes as C

import numpy as np
import pytest

import paper_2407_08330_b200 as P
from oracle import block_oracle as B


@pytest.mark.parametrize("counter, key, want", [      # known-answer vectors published with the generator
    ((0,) * 4, (0,) * 2, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
])
def test_philox_known_answers(counter, key, want):
    assert B.philox4x32(counter, key) == want


def test_keep_mask_is_kept_with_its_probability():
    D = B.keep_mask(64, 128, 12345, 6, 7, 0.25)
    n = D.size                                       # kept: binomial, four standard deviations
    assert abs((D > 0).mean() - 0.75) < 4 * np.sqrt(0.25 * 0.75 / n)
    assert set(np.unique(D)) == {0.0, 65536 / (65536 - 16384)}
    assert (D != B.keep_mask(64, 128, 12345, 6, 8, 0.25)).any() and (D != B.keep_mask(64, 128, 12345, 7, 7, 0.25)).any()


def test_layer_norm_gradient_against_differences():
    rng = np.random.default_rng(0)
    h, w, b, dy = rng.normal(size=(3, 11)), rng.normal(size=11), rng.normal(size=11), rng.normal(size=(3, 11))
    loss = lambda h, w, b: (B.layer_norm(h, w, b, 1e-5)[0] * dy).sum()
    _, mean, rstd = B.layer_norm(h, w, b, 1e-5)
    dh, dw, db = B.layer_norm_bwd(dy, h, mean, rstd, w)
    for x, g, f in ((h, dh, lambda x: loss(x, w, b)), (w, dw, lambda x: loss(h, x, b)), (b, db, lambda x: loss(h, w, x))):
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = 1e-5
            assert abs((f(x + e) - f(x - e)) / 2e-5 - g[i]) < 1e-7


A, ODD = 0x10000, 0x10002      # addresses that nothing reads: the calls below end at their checks


def _drop(x=A, res=None, rng=A, rows=4, cols=8, dtype=1, p=0.1, y=A):
    return P.lib().hdt_dropout(x, res, rng, 0, rows, cols, dtype, p, y, None)


def _fwd(x=A, res=None, w=A, b=A, rng=None, p=0.0, rows=4, cols=8, dtype=1, w_dtype=1, eps=1e-5, h=None, y=A, mean=A, rstd=A):
    return P.lib().hdt_layer_norm_fwd(x, res, w, b, rng, 0, p, rows, cols, dtype, w_dtype, eps, h, y, mean, rstd, None)


def _bwd(dy=A, h=A, mean=A, w=A, rng=None, p=0.0, rows=4, cols=8, dtype=1, w_dtype=1, dres=A, dx=None, dw=A, ws=A, n=1 << 20):
    return P.lib().hdt_layer_norm_bwd(dy, None, h, mean, A, w, rng, 0, p, rows, cols, dtype, w_dtype, dres, dx, dw, A, ws, n, None)


@pytest.mark.parametrize("call, code", [
    (lambda: _drop(rows=-1), -1), (lambda: _drop(cols=0), -1), (lambda: _drop(cols=8193), -3), (lambda: _drop(rows=2 ** 31), -3),
    (lambda: _drop(dtype=7), -3), (lambda: _drop(p=1.0), -1), (lambda: _drop(p=-0.1), -1), (lambda: _drop(p=float("nan")), -1),
    (lambda: _drop(rng=None), -1), (lambda: _drop(rng=A + 4), -1), (lambda: _drop(x=None), -1), (lambda: _drop(y=None), -1), (lambda: _drop(x=A + 1), -1),
    (lambda: _drop(dtype=0, y=ODD), -1), (lambda: _drop(rows=0, x=None, y=None), 0),
    (lambda: _fwd(w_dtype=3), -3), (lambda: _fwd(dtype=0, w_dtype=1), -3), (lambda: _fwd(eps=-1.0), -1), (lambda: _fwd(eps=float("nan")), -1),
    (lambda: _fwd(p=0.5), -1), (lambda: _fwd(p=0.5, rng=A), -1), (lambda: _fwd(p=1e-7, rng=A), -1), (lambda: _fwd(res=A), -1), (lambda: _fwd(w=None), -1), (lambda: _fwd(mean=None), -1),
    (lambda: _fwd(mean=ODD), -1), (lambda: _fwd(w_dtype=0, w=ODD), -1), (lambda: _fwd(rows=0), 0),
    (lambda: _bwd(dy=None), -1), (lambda: _bwd(dw=None), -1), (lambda: _bwd(p=0.5, rng=A), -1), (lambda: _bwd(p=1e-7, rng=A), -1), (lambda: _bwd(rows=2 ** 31 - 2 ** 15), -3), (lambda: _bwd(ws=None), -4), (lambda: _bwd(n=63), -4),
    (lambda: _bwd(ws=A + 128), -1), (lambda: _bwd(h=A + 1), -1), (lambda: _bwd(cols=9000), -3),
])
def test_refusals(call, code):
    assert call() == code
    if code:
        assert P.lib().hdt_last_error()


def test_workspace_bytes():
    assert P.hdt_layer_norm_workspace_bytes(1, 768) >= 2 * 768 * 4
    assert P.hdt_layer_norm_workspace_bytes(0, 768) >= 256
    assert P.hdt_layer_norm_workspace_bytes(-1, 768) == 0 and P.hdt_layer_norm_workspace_bytes(4, 0) == 0
