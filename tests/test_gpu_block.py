"""A decoder block made of the library's calls, as a model strings them together: dropout and norm in front of causal
self-attention with a relative bias, dropout and norm behind it, cross-attention to the encoder's anchors, with a backward
pass by hand, against the same block in 64 bits with torch's gradients."""
import numpy as np
import pytest
import torch

import gen
from gpu_util import dev_struct
from oracle import block_oracle as B, self_oracle as S

pytestmark = pytest.mark.gpu
H, D, LEVELS = 3, 64, 6
E = H * D


def attend(q, k, v, cu_q, cu_k, bias_at, seen_at):
    """softmax attention in 64 bits, document by document; bias_at, seen_at: per document."""
    out = []
    for b in range(len(cu_q) - 1):
        x, y, z = q[cu_q[b]:cu_q[b + 1]], k[cu_k[b]:cu_k[b + 1]], v[cu_k[b]:cu_k[b + 1]]
        a = torch.einsum("ihc,jhc->hij", x, y) / D ** 0.5 + bias_at(b)
        out.append(torch.einsum("hij,jhc->ihc", torch.softmax(a.masked_fill(~seen_at(b), -torch.inf), 2), z))
    return torch.cat(out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decoder_block(dtype):
    import paper_2407_08330_b200 as P
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    enc = gen.small_random_batch(3, n_seqs=2, max_len=150, K=(3, 20))
    level, _, cu_enc = dev_struct(enc)
    cu_e = enc.cu_seqlens.tolist()
    cu_d = [0, 70, 203]
    cu_q = torch.tensor(cu_d, dtype=torch.int32, device="cuda")
    T, p = cu_d[-1], 0.1
    g = torch.Generator(device="cuda").manual_seed(4)
    rn = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(dt)
    x, res, mem_k, mem_v, dout = rn(T, E), rn(T, E), rn(cu_e[-1], H, D), rn(cu_e[-1], H, D), rn(T, E)
    w1, b1, w2, b2 = rn(E), rn(E), rn(E), rn(E)
    wq, wk, wv, wc = (rn(E, E, scale=E ** -0.5) for _ in range(4))
    bias = rn(32, H)
    rng = torch.tensor([99, 7], dtype=torch.int64, device="cuda")
    h3 = lambda t: t.view(-1, H, D)

    # forward
    y1, h1, m1, r1 = P.hdt_layer_norm_fwd(x, w1, b1, residual=res, p=p, rng=rng, site=0)
    q, k, v = (h3(y1 @ w).contiguous() for w in (wq, wk, wv))
    o, lse = P.hdt_self_attn_fwd(cu_q, cu_q, q, k, v, bias=bias)
    y2, h2, m2, r2 = P.hdt_layer_norm_fwd(o.view(T, E), w2, b2, residual=h1, p=p, rng=rng, site=1)
    qc = h3(y2 @ wc).contiguous()
    oc, lsec = P.hdt_cross_attn_fwd(level, cu_enc, cu_q, LEVELS, qc, mem_k, mem_v)
    out = P.hdt_dropout(oc.view(T, E), p, rng, site=2, residual=h2)
    # backward
    doc = P.hdt_dropout(dout, p, rng, site=2)
    dqc, dmk, dmv = P.hdt_cross_attn_bwd(level, cu_enc, cu_q, LEVELS, qc, mem_k, mem_v, oc, lsec, h3(doc))
    dy2, dwc = dqc.view(T, E) @ wc.t(), y2.t() @ dqc.view(T, E)
    do, dh1, dw2, db2 = P.hdt_layer_norm_bwd(dy2, h2, m2, r2, w2, d_h=dout, p=p, rng=rng, site=1)
    dq, dk, dv, dbias = P.hdt_self_attn_bwd(cu_q, cu_q, q, k, v, o, lse, h3(do), bias=bias)
    dy1 = sum(t.view(T, E) @ w.t() for t, w in ((dq, wq), (dk, wk), (dv, wv)))
    dx, dres, dw1, db1 = P.hdt_layer_norm_bwd(dy1, h1, m1, r1, w1, d_h=dh1, p=p, rng=rng, site=0)
    P.hdt_device_status()

    # the same in 64 bits
    leaf = {n: t.double().cpu().requires_grad_() for n, t in dict(x=x, res=res, mem_k=mem_k, mem_v=mem_v, w1=w1, b1=b1, w2=w2, b2=b2, wq=wq, wk=wk, wv=wv, wc=wc, bias=bias).items()}
    L = leaf
    mask = [torch.from_numpy(B.keep_mask(T, E, 99, 7, s, p)) for s in range(3)]
    norm = lambda h, w, b: (h - h.mean(1, keepdim=True)) / torch.sqrt(h.var(1, unbiased=False, keepdim=True) + 1e-5) * w + b
    a1 = L["res"] + mask[0] * L["x"]
    z1 = norm(a1, L["w1"], L["b1"])
    dist = lambda b: np.subtract.outer(np.arange(cu_d[b + 1] - cu_d[b]), np.arange(cu_d[b + 1] - cu_d[b]))
    s1 = attend(h3(z1 @ L["wq"]), h3(z1 @ L["wk"]), h3(z1 @ L["wv"]), cu_d, cu_d, lambda b: L["bias"][torch.from_numpy(S.bucket(dist(b), 32, 128, True))].permute(2, 0, 1),
                lambda b: torch.from_numpy(dist(b) >= 0))
    a2 = a1 + mask[1] * s1.reshape(T, E)
    z2 = norm(a2, L["w2"], L["b2"])
    lev = torch.from_numpy(enc.level)
    chosen = (lev >= 0) & ((LEVELS >> lev.clamp(min=0)) & 1).bool()
    s2 = attend(h3(z2 @ L["wc"]), L["mem_k"], L["mem_v"], cu_d, cu_e, lambda b: 0.0, lambda b: chosen[cu_e[b]:cu_e[b + 1]][None, None].expand(1, cu_d[b + 1] - cu_d[b], -1))
    want = a2 + mask[2] * s2.reshape(T, E)
    want.backward(dout.double().cpu())
    got = dict(x=dx, res=dres, mem_k=dmk, mem_v=dmv, w1=dw1, b1=db1, w2=dw2, b2=db2, wc=dwc, bias=dbias,
               wq=y1.t() @ dq.view(T, E), wk=y1.t() @ dk.view(T, E), wv=y1.t() @ dv.view(T, E))
    # twenty-odd roundings of a tensor in a row, each at most half a step relative to its size; sums mix them at random
    tol = 24 * torch.finfo(dt).eps / 2 if dtype == "bf16" else 1e-4
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())
    assert rel(out, want.detach()) < tol
    for n, t in got.items():
        assert rel(t, leaf[n].grad) < tol, n
