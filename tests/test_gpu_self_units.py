"""Self-attention in the forms that calls of ordinary training size take: units of two full row tiles over many key tiles, several units to
a CTA, more documents than one turn of the preparation takes; and the correction of delta for O's rounding in bf16.

Bounds as in test_gpu_self.py (results of a few heads against the definition: a head's results depend on that head alone).  The
correction: dS' = P (dP - delta') with delta' = delta + sum_j P (dP - delta), which no longer holds the rounding of O: with D_i the bound of
that rounding's part of delta, dK and dBias are off by fp32 terms only,
  x' = P [2 e (sum_j P |dO| |V| + |delta|) + e |dO| |V_j|],
and dQ = sum_j bf16(dS) K - r sum_j bf16(P) K, where dS still has the rounding of O in it, by the rounding of that part (u P D_i) and of
P under r (u P D_i):
  dQ     u |dQ| + scale sum_j [(u + e) |dS| + 2 u P D_i + x'] |K|
  dK     u |dK| + scale sum_i [(u + e) |dS| + x'] |Q|
  dBias  u |dBias| + sum over the bucket's pairs of [e |dS| + x']."""
import copy

import numpy as np
import pytest
import torch

from oracle import self_oracle as S
from test_gpu_self import Case, f64

pytestmark = pytest.mark.gpu


def check_heads(c, got, heads):
    """c.check of some heads."""
    s = copy.copy(c)
    for n in ("q", "k", "v", "do"):
        setattr(s, n, getattr(c, n)[:, heads])
    s.bias = None if c.bias is None else c.bias[:, heads]
    s.H = len(heads)
    s.check({n: t[heads] if n == "lse" else t[:, heads] for n, t in got.items()})


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("buckets, far", [(32, 128), (64, 2000)])
def test_long_documents_on_full_units(d, causal, buckets, far):
    """22 blocks of 128 rows and 13 units of 256 a head, 16 heads: units of 256 rows are taken from 148 on."""
    H = 16
    c = Case([1500, 777, 257, 100], [1500, 900, 257, 1100], H, d, "bf16", causal, buckets, far, room=3, behind=5)
    assert sum((n + 255) // 256 for n in c.lq) * H >= 148
    check_heads(c, c.run(), [0, H - 1])


@pytest.mark.parametrize("d", [64, 128])
def test_units_of_every_length_follow_one_another(d):
    """Long units, short ones and empty ones on every CTA, 2200 of them."""
    lens = [900, 0, 1, 300, 128, 129, 640, 31, 256, 257, 5, 470] * 3
    keys = [n + (0, 60, 200)[i % 3] for i, n in enumerate(lens)]
    c = Case(lens, keys, 24, d, "bf16", True, 32, 100, behind=9)
    check_heads(c, c.run(), [11])


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_more_documents_than_a_turn_of_the_preparation(dtype, d, causal):
    """1500 documents, 1500 blocks and more of them."""
    lens = [(11 * i) % 19 + (140 if i % 97 == 0 else 0) for i in range(1500)]
    keys = [n + i % 5 if i % 7 else n // 2 for i, n in enumerate(lens)]
    assert sum(lens) > 4 * len(lens) and sum((n + 127) // 128 for n in lens) > 1024
    c = Case(lens, keys, 1, d, dtype, causal, 16, 40, room=2)
    c.check(c.run())


@pytest.mark.parametrize("dtype, rows", [("bf16", 128), ("f32", 64)])
def test_more_blocks_than_a_turn_of_the_preparation_sorts(dtype, rows):
    """Documents of 1400 blocks whose rows see no key but the last 70, so that the oracle's work stays small."""
    import paper_2407_08330_b200 as P
    c = Case([70, 100], [70, 100], 1, 64, dtype)
    n, blind = rows * 700 + 5, 2 * (rows * 700 + 5) - 70
    cu_q = torch.tensor([0, n, 2 * n, 2 * n + 100], dtype=torch.int32, device="cuda")
    cu_k = torch.tensor([0, 0, 70, 170], dtype=torch.int32, device="cuda")
    behind = lambda x: torch.cat([torch.randn(blind, 1, 64, device="cuda").to(x.dtype), x])
    q, do = behind(c.q), behind(c.do)
    o, lse = P.hdt_self_attn_fwd(cu_q, cu_k, q, c.k, c.v, bias=c.bias, out=torch.full_like(q, -7.0))
    dq, dk, dv, db = P.hdt_self_attn_bwd(cu_q, cu_k, q, c.k, c.v, o, lse, do, bias=c.bias, dq=torch.full_like(q, -7.0))
    P.hdt_device_status()
    assert not o[:blind].any() and not dq[:blind].any() and torch.isneginf(lse[:, :blind]).all()
    c.check(dict(o=o[blind:], lse=lse[:, blind:], dq=dq[blind:], dk=dk, dv=dv, dbias=db))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[7, 5], [3] * 40 + [7] * 20, [130, 200, 9]], ids=["few", "short", "longer"])
def test_rounding_of_o_leaves_delta(d, lens):
    """Values near one another and far from 0: dO . O is a large number known to bf16, dP - delta a small one.  The bounds above hold, and
    the uncorrected gradients, from the O that was stored, do not keep to them (the bias', a sum over many rows of either sign, only where
    the rows are few)."""
    import paper_2407_08330_b200 as P
    H = 3
    c = Case(lens, lens, H, d, "bf16", True, 16, 40)
    g = np.random.default_rng(d)
    base = 1 + g.integers(0, 127, (1, H, d)) / 128              # the bf16 grid of [1, 2): steps of 1/128
    c.v[:] = torch.from_numpy(base + g.integers(0, 2, (c.Tk, H, d)) / 128).cuda().bfloat16()
    for x in (c.q, c.k, c.bias):
        x.mul_(0.125)
    got = c.run()
    u, f = 2.0 ** -8, 2.0 ** -24
    want_db = loose_db = bound_db = 0.0
    beyond = dict(dq=False, dk=False, dbias=False)

    def held(name, x, want, bound, loose):
        assert (np.abs(x - want) <= bound * 1.01 + 1e-30).all(), f"{name}: worst excess {(np.abs(x - want) - bound).max():.3e}"
        beyond[name] |= bool((np.abs(loose - want) > bound).any())

    for b in range(len(lens)):
        r = slice(c.cq[b], c.cq[b + 1])
        q, k, v, do, bias, o = f64(c.q[r]), f64(c.k[r]), f64(c.v[r]), f64(c.do[r]), f64(c.bias), f64(got["o"][r])
        w = S.document(q, k, v, bias, 40, True, c.scale, do)
        p, ds, n = w["p"], np.abs(w["ds"]), lens[b]
        L = c.scale * np.einsum("ihc,jhc->hij", np.abs(q), np.abs(k)).max()
        A = 2 * L + 2 * np.abs(bias).max() + np.log(n + 1.0)
        e = f * ((d + 16) * (L + A) + n + d + 16)
        pv = np.einsum("hij,jhc->ihc", p, np.abs(v))
        D = np.einsum("ihc,ihc->hi", np.abs(do), u * np.abs(w["o"]) + (u + e) * pv)[..., None]
        x = p * (2 * e * (np.einsum("ihc,ihc->hi", np.abs(do), pv) + np.abs(np.einsum("ihc,ihc->hi", do, w["o"])))[..., None]
                 + e * np.einsum("ihc,jhc->hij", np.abs(do), np.abs(v)))
        loose = p * (w["dp"] - np.einsum("ihc,ihc->hi", do, o)[..., None])      # the gradients from the stored O, otherwise exact
        y = (u + e) * ds + x
        held("dq", f64(got["dq"][r]), w["dq"], u * np.abs(w["dq"]) + c.scale * np.einsum("hij,jhc->ihc", y + 2 * u * p * D, np.abs(k)),
             c.scale * np.einsum("hij,jhc->ihc", loose, k))
        held("dk", f64(got["dk"][r]), w["dk"], u * np.abs(w["dk"]) + c.scale * np.einsum("hij,ihc->jhc", y, np.abs(q)), c.scale * np.einsum("hij,ihc->jhc", loose, q))
        for name, z in (("bound", e * ds + x), ("loose", loose)):
            t = np.zeros_like(bias)
            np.add.at(t, w["bucket"].reshape(-1), z.transpose(1, 2, 0).reshape(-1, H))
            if name == "bound":
                bound_db = bound_db + t
            else:
                loose_db = loose_db + t
        want_db = want_db + w["dbias"]
    held("dbias", f64(got["dbias"]), want_db, u * np.abs(want_db) + bound_db, loose_db)
    assert beyond["dq"] and beyond["dk"] and (beyond["dbias"] or len(lens) > 2), beyond
