"""Sizes that do not fit the C interface's 32 bits are refused, not taken modulo 2^32 (shapes alone: no GPU)."""
import pytest
import torch

import paper_2407_08330_b200 as P

BIG = 2 ** 32 + 8      # 8, modulo 2^32
meta = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="meta")


def _self(call, tokens=8, bias=None, **kw):
    q = meta(tokens, 2, 64)
    cu = meta(3, dtype=torch.int32)
    more = () if call is P.hdt_self_attn_fwd else (q, meta(2, tokens, dtype=torch.float32), q)
    return call(cu, cu, q, q, q, *more, bias=bias, **kw)


@pytest.mark.parametrize("call", [
    lambda: P.hdt_dropout(meta(1, BIG), 0.1, meta(2, dtype=torch.int64)),
    lambda: P.hdt_layer_norm_fwd(meta(1, BIG), meta(BIG), meta(BIG)),
    lambda: P.hdt_layer_norm_bwd(meta(1, BIG), meta(1, BIG), meta(1, dtype=torch.float32), meta(1, dtype=torch.float32), meta(BIG)),
    lambda: _self(P.hdt_self_attn_fwd, tokens=BIG), lambda: _self(P.hdt_self_attn_bwd, tokens=BIG),
    lambda: _self(P.hdt_self_attn_fwd, bias=meta(BIG, 2)), lambda: _self(P.hdt_self_attn_bwd, bias=meta(BIG, 2)),
    lambda: _self(P.hdt_self_attn_fwd, bias=meta(32, 2), max_distance=2 ** 32 + 128), lambda: _self(P.hdt_self_attn_bwd, bias=meta(32, 2), max_distance=2 ** 32 + 128),
    lambda: P.hdt_self_bucket_borders(8, 2 ** 32 + 64),
])
def test_refused(call):
    with pytest.raises(P.HdtError) as e:
        call()
    assert e.value.code == -3


def test_workspace_of_such_sizes_is_none():
    assert P.hdt_layer_norm_workspace_bytes(4, 8) > 0 and P.hdt_layer_norm_workspace_bytes(4, BIG) == 0
    f = lambda *a: P.hdt_self_workspace_bytes(*a, True, torch.bfloat16, False)
    assert f(2, 8, 8, 2, 64, 32, 128) > 0
    for i in range(7):
        a = [2, 8, 8, 2, 64, 32, 128]
        a[i] += 2 ** 32
        assert f(*a) == 0, i
