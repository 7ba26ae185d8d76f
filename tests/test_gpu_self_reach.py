"""What a row that is not finite reaches in the fp32 kernels and in a step of decoding: the rows that see it, and no other.
The rest of a call's results are compared with those of the same call on finite rows, bit by bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BAD = [float("nan"), float("inf")]


def tensors(T, Tk, H, d, dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = lambda n: torch.randn(n, H, d, generator=g, device="cuda").to(dtype)
    return t(T), t(Tk), t(Tk), t(T), torch.randn(32, H, generator=g, device="cuda").to(dtype)


def cu(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("n, nk, at", [(200, 200, 0), (200, 200, 63), (200, 200, 64), (200, 200, 100), (200, 200, 127), (200, 200, 199), (70, 203, 150), (70, 203, 134), (33, 33, 5)])
def test_key_row_reaches_the_rows_that_see_it(d, bad, with_bias, n, nk, at):
    """Causal: key `at` is seen from row at - (nk - n) on."""
    import paper_2407_08330_b200 as P
    q, k, v, do, bias = tensors(n, nk, 2, d)
    bias = bias if with_bias else None
    a = (cu(0, n), cu(0, nk))
    o, lse = P.hdt_self_attn_fwd(*a, q, k, v, bias=bias)
    dq = P.hdt_self_attn_bwd(*a, q, k, v, o, lse, do, bias=bias)[0]
    first = max(0, at - (nk - n))
    for both in (True, False):      # K and V, or V alone
        k1, v1 = k.clone(), v.clone()
        v1[at] = bad
        if both:
            k1[at] = bad
        o1, lse1 = P.hdt_self_attn_fwd(*a, q, k1, v1, bias=bias)
        assert torch.equal(o1[:first], o[:first]) and torch.equal(lse1[:, :first], lse[:, :first])
        assert not o1[first:].isfinite().any()
        dq1, dk1, dv1, _ = P.hdt_self_attn_bwd(*a, q, k1, v1, o1, lse1, do, bias=bias)
        assert torch.equal(dq1[:first], dq[:first])
    P.hdt_device_status()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("n, nk, at", [(200, 200, 0), (200, 200, 63), (200, 200, 64), (200, 200, 100), (200, 200, 199), (70, 203, 17), (70, 203, 69), (33, 33, 5)])
def test_query_row_reaches_the_keys_that_it_sees(d, bad, with_bias, n, nk, at):
    import paper_2407_08330_b200 as P
    q, k, v, do, bias = tensors(n, nk, 2, d, seed=1)
    bias = bias if with_bias else None
    a = (cu(0, n), cu(0, nk))
    o, lse = P.hdt_self_attn_fwd(*a, q, k, v, bias=bias)
    dq, dk, dv, _ = P.hdt_self_attn_bwd(*a, q, k, v, o, lse, do, bias=bias)
    last = at + (nk - n)            # the last key that the row sees
    others = [i for i in range(n) if i != at]
    q1, do1 = q.clone(), do.clone()
    q1[at] = do1[at] = bad
    o1, lse1 = P.hdt_self_attn_fwd(*a, q1, k, v, bias=bias)
    assert torch.equal(o1[others], o[others]) and torch.equal(lse1[:, others], lse[:, others])
    for o2, lse2 in ((o1, lse1), (o, lse)):
        dq1, dk1, dv1, _ = P.hdt_self_attn_bwd(*a, q1, k, v, o2, lse2, do1, bias=bias)
        assert torch.equal(dk1[last + 1:], dk[last + 1:]) and torch.equal(dv1[last + 1:], dv[last + 1:])
        assert torch.equal(dq1[others], dq[others])
    P.hdt_device_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("keys", [4, 37, 900])
def test_step_of_several_rows(dtype, d, bad, keys):
    """Four and three rows of two documents: the last keys are seen by the last rows only."""
    import paper_2407_08330_b200 as P
    q, k, v, _, bias = tensors(7, keys + 50, 3, d, dtype, seed=2)
    a = (cu(0, 4, 7), cu(0, keys, keys + 50))
    o, lse = P.hdt_self_attn_fwd(*a, q, k, v, bias=bias)
    for back in range(3):           # the key that only the last `back` + 1 rows see
        k1, v1 = k.clone(), v.clone()
        for end in (keys, keys + 50):
            k1[end - 1 - back] = v1[end - 1 - back] = bad
        o1, lse1 = P.hdt_self_attn_fwd(*a, q, k1, v1, bias=bias)
        clean = list(range(0, 3 - back)) + list(range(4, 6 - back))
        assert torch.equal(o1[clean], o[clean]) and torch.equal(lse1[:, clean], lse[:, clean])
        assert not o1[[i for i in range(7) if i not in clean]].isfinite().any()
    P.hdt_device_status()
