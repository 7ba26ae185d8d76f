"""The caller's buffers for the gradients of the layer norm."""
import pytest
import torch

import paper_2407_08330_b200 as P

A = 0x10000      # an address that nothing reads: the calls with it end at their checks


def _bwd(p, dres, dx, rng=A):
    return P.lib().hdt_layer_norm_bwd(A, None, A, A, A, A, rng, 0, p, 4, 8, 1, 1, dres, dx, A, A, A, 1 << 20, None)


def test_one_buffer_for_two_gradients_is_refused():
    """With dropout d_x and d_residual differ."""
    assert _bwd(0.5, A, A) == -1 and b"d_x" in P.lib().hdt_last_error()
    assert _bwd(1e-7, A, A) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("rows, cols, dtype", [(9, 64, torch.float32), (33, 768, torch.bfloat16), (5, 1021, torch.float32), (7, 2048, torch.bfloat16), (3, 5000, torch.bfloat16)])
@pytest.mark.parametrize("with_dh", [False, True])
def test_gradient_of_x_is_written_without_dropout(rows, cols, dtype, with_dh):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, dy, dh = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(3))
    w, b = (torch.randn(cols, generator=g, device="cuda") for _ in range(2))
    dh = dh if with_dh else None
    _, h, mean, rstd = P.hdt_layer_norm_fwd(x, w, b)
    want, want_res, want_w, want_b = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh)
    assert want is want_res
    dx, dres = torch.full_like(x, 7.0), torch.full_like(x, 8.0)
    got, got_res, got_w, got_b = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh, d_x=dx, d_residual=dres)
    assert got is dx and got_res is dres
    for y, z in ((dx, want), (dres, want), (got_w, want_w), (got_b, want_b)):
        assert torch.equal(y, z)
    dx.fill_(7.0)
    got, got_res, _, _ = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh, d_x=dx)      # the one that is not given is made
    assert got is dx and torch.equal(got, want) and torch.equal(got_res, want)
    dx.fill_(7.0)
    got, got_res, _, _ = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=dh, d_x=dx, d_residual=dx)      # both in one buffer
    assert got is dx and got_res is dx and torch.equal(dx, want)
    if with_dh:                                                                                          # in place of d_h
        in_place = dh.clone()
        got, got_res, _, _ = P.hdt_layer_norm_bwd(dy, h, mean, rstd, w, d_h=in_place, d_x=in_place)
        assert got is in_place and torch.equal(got, want) and torch.equal(got_res, want)
