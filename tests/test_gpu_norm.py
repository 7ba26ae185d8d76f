"""Dropout and layer norm on the GPU against the 64-bit definitions.

Bounds.  An output is rounded once to its type (eps / 2 of the value).  Before that, fp32: a sum over n columns is
at most 32 additions in a row on a lane (four chunks of eight) and ten more between lanes and warps, so it is off by less
than 64 x 2^-24 of the sum of magnitudes; every other step is a few roundings of 2^-24.  With M = the largest |h| of the
row, the quantities that a row's result is a sum of are bounded by the `size` arrays below; twice 64 x 2^-24 of them
covers mean, variance and the products (rsqrt and the reciprocal of n are good to 2 units in the last place).  Column
sums: at most `rows / 4` additions in a row on a lane in the longest walk here (the grid holds all rows of these cases in
one to a few steps), bounded by (64 + rows) x 2^-24 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
T = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(x, dtype):
    t = torch.from_numpy(np.asarray(x, np.float64)).to(T[dtype]).cuda()
    return t, t.double().cpu().numpy()


def state(seed=0x123456789ABCDEF, offset=5):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda"), seed, offset


def near(got, want, fp32, what):
    half = torch.finfo(got.dtype).eps / 2
    got = got.double().cpu().numpy()
    bound = half * np.abs(want) + fp32 * (1 + half) + 1e-37
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), f"{what}: worst excess {over.max():.3e} at {np.unravel_index(over.argmax(), over.shape)}"


SHAPES = [(1, 1), (1, 8), (5, 7), (3, 24), (9, 33), (33, 64), (7, 100), (17, 128), (4, 250), (6, 256), (5, 511), (130, 768), (3, 1021), (9, 1024), (2, 1031),
          (3, 2048), (2, 3001), (2, 4096), (2, 5000), (1, 8192), (1, 8191)]


@pytest.mark.parametrize("rows, cols", SHAPES)
@pytest.mark.parametrize("dtype, w_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("p, res", [(0.0, False), (0.0, True), (0.1, True), (0.37, False)])
def test_layer_norm(rows, cols, dtype, w_dtype, p, res):
    import paper_2407_08330_b200 as P
    g = np.random.default_rng(rows * 10007 + cols)
    x, x_ = dev(g.normal(size=(rows, cols)) * 2 + 0.5, dtype)
    r, r_ = dev(g.normal(size=(rows, cols)), dtype)
    w, w_ = dev(g.normal(size=cols) * 0.3 + 1, w_dtype)
    b, b_ = dev(g.normal(size=cols), w_dtype)
    rng, seed, offset = state()
    D = B.keep_mask(rows, cols, seed, offset, 3, p) if p else 1.0
    y, h, mean, rstd = P.hdt_layer_norm_fwd(x, w, b, residual=r if res else None, p=p, rng=rng, site=3)
    h_ = x_ * D + (r_ if res else 0.0)
    y_, mean_, rstd_ = B.layer_norm(h_, w_, b_, 1e-5)
    M = np.abs(h_).max(1) + 1e-30
    near(h, h_, 4 * U * (np.abs(x_) * 2 + np.abs(r_)), "h")
    near(mean, mean_, 128 * U * M, "mean")
    # var is off by 128 U (M^2 at most per column, twice): relative to var + eps, half of it in rstd
    off = 128 * U * (1 + 2 * M * M * rstd_ ** 2)
    near(rstd, rstd_, off * rstd_, "rstd")
    size = (np.abs(h_) + 2 * M[:, None]) * rstd_[:, None] * np.abs(w_) * (1 + 2 * (M * rstd_)[:, None] ** 2) + np.abs(b_)
    near(y, y_, 128 * U * size, "y")
    # backward, from the rounded h and the statistics that the forward left
    dy, dy_ = dev(g.normal(size=(rows, cols)), dtype)
    dh, dh_ = dev(g.normal(size=(rows, cols)), dtype)
    hr, m32, r32 = (t.double().cpu().numpy() for t in (h, mean, rstd))
    dx, dres, dw, db = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh if res else None, p=p, rng=rng, site=3)
    dres_, dw_, db_ = B.layer_norm_bwd(dy_, hr, m32, r32, w_, dh_ if res else None)
    xh = (np.abs(hr) + np.abs(m32)[:, None]) * r32[:, None]
    gw = np.abs(dy_ * w_)
    size = r32[:, None] * (gw + gw.mean(1, keepdims=True) + xh * (gw * xh).mean(1, keepdims=True)) + np.abs(dh_)
    near(dres, dres_, 128 * U * size, "d_residual")
    near(dx, dres_ * D, 130 * U * size * (1 / (1 - p)), "d_x")
    near(dw, dw_, (64 + rows) * U * (np.abs(dy_) * xh).sum(0), "d_weight")
    near(db, db_, (64 + rows) * U * np.abs(dy_).sum(0), "d_bias")
    if p == 0:
        assert dx is dres
        if not res:
            assert h is x


@pytest.mark.parametrize("rows, cols", SHAPES + [(57, 768), (300, 16), (2000, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("p, res", [(0.1, True), (0.5, False), (0.0, True), (0.9999999, False)])
def test_dropout(rows, cols, dtype, p, res):
    import paper_2407_08330_b200 as P
    if rows * cols > 60000:
        rows = max(1, 60000 // cols)
    g = np.random.default_rng(rows + cols)
    x, x_ = dev(g.normal(size=(rows, cols)), dtype)
    r, r_ = dev(g.normal(size=(rows, cols)), dtype)
    rng, seed, offset = state(-7, 2 ** 40 + 9)
    D = B.keep_mask(rows, cols, seed, offset, 2 ** 31 - 1, p)
    y = P.hdt_dropout(x, p, rng, site=2 ** 31 - 1, residual=r if res else None)
    want = x_ * D + (r_ if res else 0)
    near(y, want, 4 * U * (np.abs(x_) * D + np.abs(r_)), "y")
    if not res:
        assert ((y == 0).cpu().numpy() == (x_ * D == 0)).all()
        # the gradient: the same mask
        d = P.hdt_dropout(torch.ones_like(x), p, rng, site=2 ** 31 - 1)
        assert ((d != 0).cpu().numpy() == (D != 0)).all()


def test_unaligned_rows_get_the_same_values():
    """A tensor one element off 16 bytes takes the scalar form: the same mask and bits of h, y up to the order of sums."""
    import paper_2407_08330_b200 as P
    rng, _, _ = state()
    n = 5 * 768
    base = torch.randn(n + 1, device="cuda").bfloat16()
    x = base[1:].view(5, 768)
    assert x.data_ptr() % 16 and x.is_contiguous()
    w, b = torch.ones(768, device="cuda").bfloat16(), torch.zeros(768, device="cuda").bfloat16()
    y, h, mean, rstd = P.hdt_layer_norm_fwd(x, w, b, p=0.3, rng=rng)
    y2, h2, mean2, rstd2 = P.hdt_layer_norm_fwd(x.clone(), w, b, p=0.3, rng=rng)
    assert torch.equal(h, h2) and torch.equal(P.hdt_dropout(x, 0.3, rng), h2)
    assert (y.float() - y2.float()).abs().max() <= 2 ** -8 * 4 * 4      # |y| < 16: one step of bf16 at most
    assert torch.allclose(mean, mean2, atol=1e-6) and torch.allclose(rstd, rstd2, rtol=1e-5)


def test_in_place_and_repeated_calls_give_the_same_bits():
    import paper_2407_08330_b200 as P
    rng, _, _ = state()
    x, r = (torch.randn(700, 768, device="cuda").bfloat16() for _ in range(2))
    w, b = torch.randn(768, device="cuda"), torch.randn(768, device="cuda")
    y, h, mean, rstd = P.hdt_layer_norm_fwd(x, w, b, residual=r, p=0.1, rng=rng)
    x2, r2 = x.clone(), r.clone()
    y2, h2, _, _ = P.hdt_layer_norm_fwd(x2, w, b, residual=r2, p=0.1, rng=rng, h=r2, out=x2)
    assert h2 is r2 and torch.equal(h, r2) and torch.equal(y, x2)
    dy, dh = (torch.randn(700, 768, device="cuda").bfloat16() for _ in range(2))
    first = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh, p=0.1, rng=rng)
    dh2 = dh.clone()
    again = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh2, p=0.1, rng=rng, d_residual=dh2)
    assert all(torch.equal(a, c) for a, c in zip(first, again))
    z = x.clone()
    assert torch.equal(P.hdt_dropout(z, 0.1, rng, residual=r, out=z), P.hdt_dropout(x, 0.1, rng, residual=r))


def test_a_p_that_rounds_to_none():
    """p below 2^-17 drops nothing; h and the gradient of x are written all the same."""
    import paper_2407_08330_b200 as P
    rng, _, _ = state()
    x, w, dy = torch.randn(5, 64, device="cuda"), torch.ones(64, device="cuda"), torch.randn(5, 64, device="cuda")
    h, dx = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    y, _, mean, rstd = P.hdt_layer_norm_fwd(x, w, w, p=1e-6, rng=rng, h=h)
    got, dres, _, _ = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, p=1e-6, rng=rng, d_x=dx)
    assert torch.equal(h, x) and got is dx and torch.equal(dx, dres) and dx is not dres


def test_rows_of_non_finite_values_stay_to_themselves():
    import paper_2407_08330_b200 as P
    x = torch.randn(9, 200, device="cuda")
    clean = P.hdt_layer_norm_fwd(x, torch.ones(200, device="cuda"), torch.zeros(200, device="cuda"))[0]
    x[4, 17], x[6, 3] = float("inf"), float("nan")
    y = P.hdt_layer_norm_fwd(x, torch.ones(200, device="cuda"), torch.zeros(200, device="cuda"))[0]
    ok = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(y[ok], clean[ok]) and y[4].isnan().any() and y[6].isnan().all()


def test_no_rows():
    import paper_2407_08330_b200 as P
    x = torch.empty(0, 768, device="cuda")
    w = torch.ones(768, device="cuda")
    y, h, mean, rstd = P.hdt_layer_norm_fwd(x, w, w)
    assert y.shape == x.shape and mean.numel() == 0
    dw, db = torch.full_like(w, 9.0), torch.full_like(w, 9.0)
    P.hdt_layer_norm_bwd(x, x, mean, rstd, w, d_weight=dw, d_bias=db)
    assert not dw.any() and not db.any()
    assert P.hdt_dropout(x, 0.5, state()[0]).numel() == 0


def test_captured_graph_draws_a_new_mask_when_the_offset_moves():
    import paper_2407_08330_b200 as P
    rng, _, _ = state()
    x, w = torch.randn(64, 768, device="cuda"), torch.ones(768, device="cuda")
    dy = torch.randn_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step():
        y, h, mean, rstd = P.hdt_layer_norm_fwd(x, w, w, p=0.1, rng=rng)
        return (y, h) + P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, p=0.1, rng=rng)
    with torch.cuda.stream(s):
        step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = step()
            rng[1] += 1
    torch.cuda.synchronize()
    rng[1] = 5
    masks = []
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        rng[1] = 5 + i
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))
        masks.append(kept[1] != 0)
        rng[1] = 6 + i
    assert (masks[0] != masks[1]).any() and (masks[1] != masks[2]).any()


def test_binding_refusals():
    import paper_2407_08330_b200 as P
    x, w = torch.randn(4, 8, device="cuda"), torch.ones(8, device="cuda")
    rng, _, _ = state()
    for call in (lambda: P.hdt_dropout(x, 0.1, None), lambda: P.hdt_dropout(x, 0.1, rng.int()), lambda: P.hdt_dropout(x.t(), 0.1, rng),
                 lambda: P.hdt_dropout(x, 0.1, rng.cpu()), lambda: P.hdt_dropout(x, 0.1, rng, residual=x[:2]), lambda: P.hdt_dropout(x.half(), 0.1, rng),
                 lambda: P.hdt_layer_norm_fwd(x, w[:4], w), lambda: P.hdt_layer_norm_fwd(x, w, w.bfloat16()), lambda: P.hdt_layer_norm_fwd(x.cpu(), w, w),
                 lambda: P.hdt_layer_norm_fwd(x, w, w, p=0.1), lambda: P.hdt_layer_norm_bwd(x, x, w, w, w)):
        with pytest.raises(P.HdtError):
            call()
