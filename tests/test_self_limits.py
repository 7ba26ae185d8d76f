"""Sizes whose work cannot be counted in 32 bits are refused (host checks; no GPU)."""
import pytest
import torch

import paper_2407_08330_b200 as P

MOST, STRIDE = 2 ** 31 - 1, 1 << 20      # the fp32 kernels walk units of both sides with a stride of up to 2^20 CTAs


@pytest.mark.parametrize("dtype, block", [(torch.float32, 64), (torch.bfloat16, 128)])
@pytest.mark.parametrize("heads", [1, 16, 4096, 65535])
@pytest.mark.parametrize("tokens", [129, 100_000])
def test_units_and_the_loops_over_them_fit_32_bits(dtype, block, heads, tokens):
    ask = lambda batch: P.hdt_self_workspace_bytes(batch, tokens, tokens, heads, 64, 0, 0, True, dtype, True)
    lo, hi = 1, 2 ** 31 - 1 - tokens                 # the largest batch that is taken
    assert ask(lo) > 0
    while hi - lo > 1:
        mid = (lo + hi) // 2
        lo, hi = (mid, hi) if ask(mid) else (lo, mid)
    assert 2 * (tokens // block + lo) * heads + STRIDE <= MOST
    assert ask(64) > 0                               # (what is in use is far from it)


def test_refusal_says_so():
    assert P.lib().hdt_self_attn_bwd(0x10000, 0x10000, None, 32764, 129, 0, 0x10000, 0x10000, 0x10000, None, 0, 0, 1, 0x10000, 0x10000, 0x10000, 0x10000, 0x10000, 0x10000,
                                     None, 65535, 64, 0, 0.0, None, 0, None) == -3
    assert b"blocks" in P.lib().hdt_last_error()
