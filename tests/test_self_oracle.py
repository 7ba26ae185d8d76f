"""Pins of the 64-bit definition of self-attention with a relative position bias, the library's bucket borders against
integer arithmetic, and what the C entry points refuse (all without a GPU)."""
import numpy as np
import pytest
import torch

import paper_2407_08330_b200 as P
from oracle import self_oracle as S


@pytest.mark.parametrize("causal", [True, False])
def test_gradients_against_differences(causal):
    rng = np.random.default_rng(1)
    nq, nk, H, d = 4, 6, 2, 3
    x = [rng.normal(size=s) for s in ((nq, H, d), (nk, H, d), (nk, H, d), (8, H))]
    do = rng.normal(size=(nq, H, d))
    loss = lambda x: (S.document(*x, 5, causal, 0.7)["o"] * do).sum()
    g = S.document(*x, 5, causal, 0.7, do)
    for n, name in enumerate(("dq", "dk", "dv", "dbias")):
        for i in np.ndindex(x[n].shape):
            y, z = [a.copy() for a in x], [a.copy() for a in x]
            y[n][i] += 1e-5
            z[n][i] -= 1e-5
            assert abs((loss(y) - loss(z)) / 2e-5 - g[name][i]) < 1e-8, (name, i)


def test_buckets_by_hand():
    # 8 buckets, exact below 4, then borders 4, 4 16^(1/4) = 8, 16, 32: exact powers of two
    assert S.borders(8, 64) == [0, 1, 2, 3, 4, 8, 16, 32]
    assert P.hdt_self_bucket_borders(8, 64) == [0, 1, 2, 3, 4, 8, 16, 32]
    assert list(S.bucket(np.array([-9, 0, 3, 7, 8, 63, 64, 10 ** 6]), 8, 64, True)) == [0, 0, 3, 4, 5, 7, 7, 7]
    assert list(S.bucket(np.array([-9, -1, 0, 1, 9]), 8, 64, False)) == [4 + 2, 5, 0, 1, 2]


def test_borders_against_integer_arithmetic():
    """The library compares logarithms, and prime factors where they are too close; many borders here are whole numbers."""
    for n in (2, 3, 4, 5, 8, 9, 16, 31, 32, 48, 64, 127, 128):
        for far in sorted({n // 2 + 1, n, 2 * n, 64, 100, 127, 128, 256, 500, 729, 1000, 1024, 2000, 4096, 6561, 10000, 16384, 31250, 32768}):
            if n // 2 < far:
                assert P.hdt_self_bucket_borders(n, far) == S.borders(n, far), (n, far)
    for n in (16, 32):
        for far in range(n, 1200, 7):
            assert P.hdt_self_bucket_borders(n, far) == S.borders(n, far), (n, far)
            assert P.hdt_self_bucket_borders(2 * n, far, False) == S.borders(n, far)


def test_row_without_keys():
    w = S.document(np.ones((3, 1, 2)), np.ones((1, 1, 2)), np.ones((1, 1, 2)), None, 0, True, 1.0, np.ones((3, 1, 2)))
    assert np.isneginf(w["lse"][0, :2]).all() and not w["o"][:2].any() and not w["dq"][:2].any()


A = 0x10000      # an address that nothing reads: the calls below end at their checks


def _fwd(cq=A, ck=A, B=2, Tq=100, Tk=100, q=A, k=A, v=A, bias=A, n=32, far=128, causal=1, o=A, lse=A, H=2, d=64, dtype=1, ws=A, ws_n=1 << 24):
    return P.lib().hdt_self_attn_fwd(cq, ck, None, B, Tq, Tk, q, k, v, bias, n, far, causal, o, lse, H, d, dtype, 0.0, ws, ws_n, None)


def _bwd(B=2, Tq=100, Tk=100, q=A, bias=A, n=32, far=128, lse=A, do=A, dq=A, dk=A, db=A, H=2, d=64, dtype=1, ws=A, ws_n=1 << 24):
    return P.lib().hdt_self_attn_bwd(A, A, None, B, Tq, Tk, q, A, A, bias, n, far, 1, A, lse, do, dq, dk, A, db, H, d, dtype, 0.0, ws, ws_n, None)


@pytest.mark.parametrize("call, code", [
    (lambda: _fwd(B=-1), -1), (lambda: _fwd(Tq=-1), -1), (lambda: _fwd(Tk=-1), -1), (lambda: _fwd(H=0), -1), (lambda: _fwd(d=96), -3), (lambda: _fwd(dtype=2), -3),
    (lambda: _fwd(H=70000), -3), (lambda: _fwd(Tq=2 ** 31 - 1, Tk=2 ** 31 - 1), -3), (lambda: _fwd(n=129), -3), (lambda: _fwd(n=1), -1), (lambda: _fwd(n=0), -1),
    (lambda: _fwd(n=33, causal=0), -1), (lambda: _fwd(n=2, causal=0), -1), (lambda: _fwd(far=16), -1), (lambda: _fwd(far=32769), -3),
    (lambda: _fwd(ws=None), -4), (lambda: _fwd(ws_n=100), -4), (lambda: _fwd(ws=A + 16), -1), (lambda: _fwd(cq=None), -1), (lambda: _fwd(ck=None), -1),
    (lambda: _fwd(q=None), -1), (lambda: _fwd(k=A + 8), -1), (lambda: _fwd(o=None), -1), (lambda: _fwd(lse=None), -1), (lambda: _fwd(bias=A + 1), -1),
    (lambda: _fwd(Tq=0, q=None, o=None), 0), (lambda: _fwd(B=0), 0),
    (lambda: _bwd(db=None), -1), (lambda: _bwd(db=A + 1), -1), (lambda: _bwd(do=None), -1), (lambda: _bwd(dq=A + 4), -1), (lambda: _bwd(dk=None), -1), (lambda: _bwd(lse=None), -1),
    (lambda: _bwd(ws_n=P.hdt_self_workspace_bytes(2, 100, 100, 2, 64, 32, 128, True, torch.bfloat16, True) - 1), -4), (lambda: _bwd(n=200), -3),
    (lambda: P.lib().hdt_self_bucket_borders(0, 128, 1, None), -1), (lambda: P.lib().hdt_self_bucket_borders(300, 1280, 1, (P.binding.C.c_int32 * 300)()), -3),
])
def test_refusals(call, code):
    assert call() == code
    if code:
        assert P.lib().hdt_last_error()


def test_workspace_bytes():
    f = lambda *a, bwd=0, dtype=torch.bfloat16: P.hdt_self_workspace_bytes(*a, True, dtype, bwd)
    assert f(4, 4096, 4096, 12, 64, 32, 128) > 0 and f(4, 4096, 4096, 12, 96, 32, 128) == 0
    assert f(4, 4096, 4096, 12, 64, 32, 128, bwd=1) > f(4, 4096, 4096, 12, 64, 32, 128) > f(4, 4096, 4096, 12, 64, 0, 0)
    # a step of decoding holds partial rows only; they grow with the keys' pieces and not with keys x rows
    assert f(8, 8, 8 * 4096, 12, 64, 32, 128) < 8 << 20
    assert f(128, 512, 128 * 4096, 12, 64, 32, 128) < 64 << 20
