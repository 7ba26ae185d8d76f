"""Offsets that describe the same rows over and over: what the documents have together passes 32 bits, and nothing outside the tensors
and the workspace is touched."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, block, docs", [(torch.bfloat16, 128, 140_000), (torch.float32, 64, 40_000)])
def test_blocks_of_overlapping_documents_beyond_32_bits(dtype, block, docs):
    """Every second document is all rows; none has a key."""
    import paper_2407_08330_b200 as P
    T = 8_000_000
    assert docs // 2 * (T // (2 * block if dtype == torch.bfloat16 else block)) > 2 ** 31 and T > 4 * docs      # (the forward's blocks; no step of decoding)
    cu_q = torch.from_numpy(np.resize(np.array([0, T], np.int32), docs + 1)).cuda()
    cu_k = torch.zeros(docs + 1, dtype=torch.int32, device="cuda")
    q, none = torch.ones(T, 1, 64, dtype=dtype, device="cuda"), torch.empty(0, 1, 64, dtype=dtype, device="cuda")
    bias = torch.zeros(32, 1, dtype=dtype, device="cuda")
    guard, marks = 1 << 20, []

    def workspace(bwd):
        n = P.hdt_self_workspace_bytes(docs, T, 0, 1, 64, 32, 128, True, dtype, bwd)
        w = torch.full((guard + n + guard,), 0x5a, dtype=torch.uint8, device="cuda")
        marks.append((w, n))
        return w[guard:guard + n]
    o, lse = P.hdt_self_attn_fwd(cu_q, cu_k, q, none, none, bias=bias, out=torch.full_like(q, -7.0), workspace=workspace(False))
    P.hdt_device_status()
    assert ((o == 0) | (o == -7)).all() and (o[:2 * block] == 0).all()
    dq, _, _, db = P.hdt_self_attn_bwd(cu_q, cu_k, q, none, none, torch.zeros_like(q), torch.full_like(lse, -torch.inf), q, bias=bias, dq=torch.full_like(q, -7.0),
                                       workspace=workspace(True))
    P.hdt_device_status()
    assert ((dq == 0) | (dq == -7)).all() and (dq[:block] == 0).all() and not db.any()
    for w, n in marks:
        assert (w[:guard] == 0x5a).all() and (w[guard + n:] == 0x5a).all()
