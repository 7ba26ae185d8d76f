"""Layer norm of more rows than the backward's grid holds at once: every CTA walks three rows and more (groups of rows), the last
trip ragged, in each of the kernel's row layouts.  Rows held at once, 148 SMs: 148 x CTAs of an SM x rows of a CTA.

Bounds (U = 2^-24) as in test_gpu_norm.py, but for the column sums: a lane adds one row a trip (at most 9 trips here), then come at most
5 additions over a warp's row groups, 3 over the warps, 33 over the partial rows and 5 over the warps of the last sum: 55 roundings, and 4 of
xhat and its product, each relative to at most the sum of magnitudes: 64 U of it."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B
from test_gpu_norm import U, dev, near, state

LAYOUTS = [      # rows, columns, types of rows and weights, rows at once
    (40007, 64, "bf16", "f32", 148 * 5 * 16), (71111, 32, "f32", "f32", 148 * 5 * 32), (20003, 128, "bf16", "bf16", 148 * 5 * 8), (9001, 250, "bf16", "bf16", 148 * 5 * 4),
    (6001, 500, "f32", "f32", 148 * 3 * 4), (6029, 768, "bf16", "f32", 148 * 3 * 4), (3500, 1024, "bf16", "bf16", 148 * 7), (2603, 1021, "f32", "f32", 148 * 5),
    (2600, 1024, "f32", "f32", 148 * 5), (2599, 771, "bf16", "bf16", 148 * 5), (1501, 2048, "bf16", "f32", 148 * 3), (1400, 1500, "f32", "f32", 148 * 3),
    (503, 4096, "bf16", "bf16", 148), (450, 5001, "f32", "f32", 148), (511, 8192, "bf16", "f32", 148)]


def keep_mask(rows, cols, seed, offset, site, p):
    """block_oracle.keep_mask on arrays."""
    m = np.uint64(0xFFFFFFFF)
    a = np.broadcast_to(np.arange((cols + 7) // 8, dtype=np.uint64)[None, :], (rows, (cols + 7) // 8))
    b = np.broadcast_to(np.arange(rows, dtype=np.uint64)[:, None], a.shape)
    c, d = np.full(a.shape, site & 0xFFFFFFFF, np.uint64), np.full(a.shape, offset & 0xFFFFFFFF, np.uint64)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    s = np.uint64(32)
    for _ in range(10):
        x, y = np.uint64(0xD2511F53) * a, np.uint64(0xCD9E8D57) * c
        a, b, c, d = (y >> s) ^ b ^ np.uint64(k0), y & m, (x >> s) ^ d ^ np.uint64(k1), x & m
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    half = np.stack([w >> np.uint64(16 * i) & np.uint64(0xFFFF) for w in (a, b, c, d) for i in (0, 1)], 2).reshape(rows, -1)[:, :cols]
    t = B.threshold(p)
    return np.where(half >= t, 65536.0 / (65536 - t), 0.0)


def test_mask_on_arrays():
    for rows, cols, site, p in ((5, 24, 3, 0.1), (3, 13, 2 ** 31 - 1, 0.6)):
        assert np.array_equal(keep_mask(rows, cols, 0x123456789ABCDEF, 5, site, p), B.keep_mask(rows, cols, 0x123456789ABCDEF, 5, site, p))


@pytest.mark.gpu
@pytest.mark.parametrize("rows, cols, dtype, w_dtype, at_once", LAYOUTS)
@pytest.mark.parametrize("p, with_dh", [(0.0, False), (0.1, True)])
def test_rows_beyond_the_grid(rows, cols, dtype, w_dtype, at_once, p, with_dh):
    import paper_2407_08330_b200 as P
    assert 3 * at_once < rows <= 9 * at_once and rows % at_once
    g = np.random.default_rng(rows + cols)
    x, x_ = dev(g.normal(size=(rows, cols)) * 2 + 0.5, dtype)
    w, w_ = dev(g.normal(size=cols) * 0.3 + 1, w_dtype)
    b, b_ = dev(g.normal(size=cols), w_dtype)
    rng, seed, offset = state()
    D = keep_mask(rows, cols, seed, offset, 3, p) if p else 1.0
    y, h, mean, rstd = P.hdt_layer_norm_fwd(x, w, b, p=p, rng=rng, site=3)
    h_ = x_ * D
    near(h, h_, 4 * U * np.abs(x_) * 2, "h")
    y_, mean_, rstd_ = B.layer_norm(h_, w_, b_, 1e-5)
    M = np.abs(h_).max(1) + 1e-30
    near(mean, mean_, 128 * U * M, "mean")
    near(rstd, rstd_, 128 * U * (1 + 2 * M * M * rstd_ ** 2) * rstd_, "rstd")
    size = (np.abs(h_) + 2 * M[:, None]) * rstd_[:, None] * np.abs(w_) * (1 + 2 * (M * rstd_)[:, None] ** 2) + np.abs(b_)
    near(y, y_, 128 * U * size, "y")
    dy, dy_ = dev(g.normal(size=(rows, cols)), dtype)
    dh, dh_ = dev(g.normal(size=(rows, cols)), dtype) if with_dh else (None, 0.0)
    hr, m32, r32 = (t.double().cpu().numpy() for t in (h, mean, rstd))
    first = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh, p=p, rng=rng, site=3)
    dx, dres, dw, db = first
    dres_, dw_, db_ = B.layer_norm_bwd(dy_, hr, m32, r32, w_, dh_ if with_dh else None)
    xh = (np.abs(hr) + np.abs(m32)[:, None]) * r32[:, None]
    gw = np.abs(dy_ * w_)
    size = r32[:, None] * (gw + gw.mean(1, keepdims=True) + xh * (gw * xh).mean(1, keepdims=True)) + np.abs(dh_)
    near(dres, dres_, 128 * U * size, "d_residual")
    near(dx, dres_ * D, 130 * U * size * (1 / (1 - p)), "d_x")
    near(dw, dw_, 64 * U * (np.abs(dy_) * xh).sum(0), "d_weight")
    near(db, db_, 64 * U * np.abs(dy_).sum(0), "d_bias")
    for _ in range(2):
        again = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh, p=p, rng=rng, site=3)
        assert all(torch.equal(s, t) for s, t in zip(first, again))
