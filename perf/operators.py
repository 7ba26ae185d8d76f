"""The operators of an encoder-decoder block around the hierarchical attention, as cases that can be timed.

Three operators, each in the form in which a block of the model calls it:

  drop   hdt_dropout: y = residual + D o x, D the scaled keep mask of a counter-based generator.  A row of
         eight columns takes one 128-bit block of Philox-4x32-10 with key = the 64-bit seed and counter =
         (column / 8, row, site, offset); column c keeps its value if the c-th 16-bit half word of the block is at
         least t = round(65536 p), and is then multiplied by 65536 / (65536 - t).
  norm   hdt_layer_norm_fwd / _bwd: h = residual + D o x, y = (h - mean) rstd weight + bias; backward with the
         reductions over the rows that the gradients of weight and bias are.
  self   hdt_self_attn_fwd / _bwd: the decoder's self-attention (or, not causal, a dense encoder's) over packed
         documents, with a learned bias per head for each bucket of relative positions, and its gradient.  The rows of
         q are the last ones of their document; with one row each this is a step of autoregressive decoding, over
         a cache whose documents have room behind their last key.

`run` has two forms of each: elementary torch operations in 32 bits, and the calls of the library (`own`).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(rows, cols, dtype, w_dtype, p, residual, backward):
    return dict(kind="norm", rows=rows, cols=cols, dtype=dtype, w_dtype=w_dtype, p=p, residual=residual, backward=backward)


def _drop(rows, cols, dtype, p, residual):
    return dict(kind="drop", rows=rows, cols=cols, dtype=dtype, p=p, residual=residual)


def _self(docs, batch, length, heads, head_dim, dtype, backward, causal=True, buckets=32, max_distance=128, rows=0):
    return dict(kind="self", docs=docs, batch=batch, length=length, heads=heads, head_dim=head_dim, dtype=dtype, backward=backward,
                causal=causal, buckets=buckets, max_distance=max_distance, rows=rows)


def listed():
    return [
        # a decoding step of eight documents: the block's residual sum and norm, latency alone
        dict(name="norm_8x768_bf16_fwd", **_norm(8, 768, "bf16", "bf16", 0.0, True, False)),
        # the junction of two sub-layers in training, at configuration 3's 4 x 8192 tokens: dropout, residual sum, norm
        dict(name="norm_drop_32768x768_bf16_fwd", **_norm(32768, 768, "bf16", "f32", 0.1, True, False)),
        # its backward pass
        dict(name="norm_drop_32768x768_bf16_bwd", **_norm(32768, 768, "bf16", "f32", 0.1, True, True)),
        # fp32, an odd number of rows and columns
        dict(name="norm_3001x1021_f32_bwd", **_norm(3001, 1021, "f32", "f32", 0.0, False, True)),
        # dropout alone (embeddings) on configuration 1's 57 tokens
        dict(name="drop_57x768_f32", **_drop(57, 768, "f32", 0.1, False)),
        # dropout and residual sum on the tokens of a batch of 2 x 32768 documents, the widest ordinary model
        dict(name="drop_65536x1024_bf16", **_drop(65536, 1024, "bf16", 0.1, True)),
        # summaries of a training batch: short decoder documents of uneven lengths
        dict(name="self_train_16x512_uneven", **_self("uneven", 16, 512, 12, 64, "bf16", True)),
        # training on long outputs
        dict(name="self_train_4x4096", **_self("full", 4, 4096, 12, 64, "bf16", True)),
        # the same with heads of 128, odd and uneven lengths, buckets that reach far
        dict(name="self_train_6x3001_d128", **_self("uneven", 6, 3001, 16, 128, "bf16", True, True, 64, 1000)),
        # a dense encoder layer over one long document, both directions
        dict(name="self_fwd_1x16384_both", **_self("full", 1, 16384, 12, 64, "bf16", False, False)),
        # training in fp32
        dict(name="self_train_2x777_f32", **_self("uneven", 2, 777, 12, 64, "f32", True)),
        # one step of autoregressive decoding
        dict(name="self_decode_8x4096", **_self("cache", 8, 4096, 12, 64, "bf16", False, True, 32, 128, 1)),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    what = rng.choice(["norm", "norm", "drop", "train", "train", "fwd", "f32", "cache"])
    if what in ("norm", "drop"):
        cols = rng.choice([_log(rng, 8, 2048), rng.choice([512, 768, 1024]), 8 * rng.randint(8, 256)])
        rows = _log(rng, 1, max(1, 32768 * 768 // cols))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        p = rng.choice([0.0, 0.1, 0.1, 0.25])
        if what == "drop":
            return _drop(rows, cols, dtype, max(p, 0.05), rng.random() < 0.6)
        return _norm(rows, cols, dtype, rng.choice([dtype, "f32"]), p, p > 0 or rng.random() < 0.5, rng.random() < 0.6)
    heads, d = rng.choice([(12, 64), (12, 64), (8, 64), (16, 128), (6, 128), (3, 64)])
    causal, buckets, far = rng.random() < 0.75, rng.choice([32, 32, 16, 64]), rng.choice([128, 128, 64, 500, 2000])
    if what == "train":
        length = _log(rng, 16, 4096)
        return _self(rng.choice(["full", "uneven"]), _log(rng, 1, max(1, min(32, 8192 // length))), length, heads, d, "bf16", True, causal, buckets, far)
    if what == "fwd":
        length = _log(rng, 16, 8192)
        return _self(rng.choice(["full", "uneven"]), _log(rng, 1, max(1, min(32, 16384 // length))), length, heads, d, "bf16", False, causal, buckets, far)
    if what == "f32":
        length = _log(rng, 1, 1024)
        return _self(rng.choice(["full", "uneven"]), _log(rng, 1, max(1, min(16, 1600 // length))), length, rng.choice([1, 4, 12]), rng.choice([64, 64, 128]), "f32",
                     rng.random() < 0.6, causal, buckets, far)
    return _self("cache", _log(rng, 1, 32), _log(rng, 32, 8192), heads, d, rng.choice(["bf16", "bf16", "f32"]), False, True, buckets, far, rng.choice([1, 1, 1, 4]))


# ---- inputs -------------------------------------------------------------------------------------
def _lengths(case):
    """Rows of q and k of every document, and the rows that its part of the cache has: they belong to the case."""
    n, L = case["batch"], case["length"]
    pool = np.random.default_rng(1000 * n + L)
    lens = np.full(n, L) if case["docs"] == "full" else pool.integers(max(1, L // 4), L + 1, n)
    if case["docs"] == "cache":
        return np.minimum(case["rows"], lens), lens, np.full(n, L + 16)
    return lens, lens, lens


def _offsets(sizes):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)).cuda()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, dtype=dt, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=g, device=dev, dtype=torch.float32) * scale + shift).to(dtype)

    s = dict(case=case)
    if case["kind"] == "self":
        n_q, n_k, room = _lengths(case)
        H, d = case["heads"], case["head_dim"]
        Tq, Tk = int(n_q.sum()), int(room.sum())
        s["cu_q"], s["cu_k"] = _offsets(n_q), _offsets(room)
        s["len_k"] = torch.from_numpy(n_k.astype(np.int32)).cuda() if case["docs"] == "cache" else None
        s["most_q"], s["most_k"] = int(n_q.max()), int(n_k.max())
        s["q"], s["k"], s["v"] = normal(Tq, H, d), normal(Tk, H, d), normal(Tk, H, d)
        s["bias"] = normal(case["buckets"], H)
        if case["backward"]:
            s["do"] = normal(Tq, H, d)
        return s
    rows, cols = case["rows"], case["cols"]
    s["rng"] = torch.randint(0, 1 << 62, (2,), generator=g, device=dev, dtype=torch.int64)
    s["site"] = seed % 24
    if case["kind"] == "drop" or not case["backward"]:
        s["x"] = normal(rows, cols)
        s["residual"] = normal(rows, cols) if case["residual"] else None
    if case["kind"] == "norm":
        wt = DTYPES[case["w_dtype"]]
        s["weight"], s["bias"] = normal(cols, dtype=wt, scale=0.2, shift=1.0), normal(cols, dtype=wt, scale=0.2)
        if case["backward"]:
            s["h"] = normal(rows, cols, scale=1.5, shift=0.1)
            h = s["h"].double()
            s["mean"] = h.mean(1).float()
            s["rstd"] = (h.var(1, unbiased=False) + 1e-5).rsqrt().float()
            s["d_y"] = normal(rows, cols)
            s["d_h"] = normal(rows, cols) if case["residual"] else None
    return s


# ---- one pass: elementary operations --------------------------------------------------------------
def _mul_hi_lo(a, b):
    """The high and low 32 bits of a * b, for a 32-bit a and a tensor b of 32-bit values."""
    upper = a * (b >> 16) + ((a * (b & 0xFFFF)) >> 16)
    return upper >> 16, (a * b) & 0xFFFFFFFF


def _philox(c0, c1, c2, c3, k0, k1, rounds):
    if rounds == 0:
        return c0, c1, c2, c3
    h0, l0 = _mul_hi_lo(0xD2511F53, c0)
    h1, l1 = _mul_hi_lo(0xCD9E8D57, c2)
    return _philox(h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0, (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF, rounds - 1)


def _keep(s, rows, cols):
    """D: 0 or 65536 / (65536 - t), [rows, cols] in fp32."""
    t = round(65536 * s["case"]["p"])
    seed, offset = s["rng"][0], s["rng"][1] & 0xFFFFFFFF
    block = torch.arange((cols + 7) // 8, device="cuda")[None, :]
    row = torch.arange(rows, device="cuda")[:, None]
    zero = torch.zeros_like(block + row)
    w = torch.stack(_philox(block + zero, row + zero, s["site"] + zero, offset + zero, seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF, 10), -1)
    half = torch.stack((w & 0xFFFF, w >> 16), -1).reshape(rows, -1)[:, :cols]
    return (half >= t).float() * (65536 / (65536 - t))


def _plain_drop(s):
    x = s["x"]
    y = x.float() * _keep(s, *x.shape)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(x.dtype)}


def _plain_norm_fwd(s):
    x = s["x"]
    h = x.float()
    if s["case"]["p"] > 0:
        h = h * _keep(s, *x.shape)
    if s["residual"] is not None:
        h = h + s["residual"].float()
    mean = h.mean(1)
    c = h - mean[:, None]
    rstd = ((c * c).mean(1) + 1e-5).rsqrt()
    y = c * rstd[:, None] * s["weight"].float() + s["bias"].float()
    return {"y": y.to(x.dtype), "h": h.to(x.dtype), "mean": mean, "rstd": rstd}


def _plain_norm_bwd(s):
    dy, dt = s["d_y"].float(), s["d_y"].dtype
    xhat = (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dres = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["d_h"] is not None:
        dres = dres + s["d_h"].float()
    dx = dres * _keep(s, *dy.shape) if s["case"]["p"] > 0 else dres
    wt = s["weight"].dtype
    return {"dx": dx.to(dt), "dresidual": dres.to(dt), "dweight": (dy * xhat).sum(0).to(wt), "dbias": dy.sum(0).to(wt)}


def _bucket(distance, case):
    """Bucket of pos(query) - pos(key): exact below half of the range, then logarithmic up to max_distance."""
    n, far = case["buckets"], case["max_distance"]
    if case["causal"]:
        base, d = torch.zeros_like(distance), distance.clamp(min=0)
    else:
        n //= 2
        base, d = (distance < 0).long() * n, distance.abs()
    exact_part = n // 2
    # (64 bits, and a nudge far below the distance to the next border, where the quotient of logarithms is whole)
    steps = torch.log(d.clamp(min=1).double() / exact_part) / math.log(far / exact_part) * (n - exact_part)
    return base + torch.where(d < exact_part, d, (exact_part + torch.floor(steps + 1e-9).long()).clamp(max=n - 1))


def _padded(x, start, length, most):
    """Packed rows [T, H, d] as [batch, H, most, d] in fp32, zero behind a document's end."""
    at = torch.arange(most, device="cuda")[None, :]
    inside = at < length[:, None]
    rows = x[(start[:, None] + at).clamp(max=x.shape[0] - 1).long()].float()
    return torch.where(inside[:, :, None, None], rows, 0.0).transpose(1, 2), inside


def _packed(x, inside, dtype):
    return x.transpose(1, 2)[inside].to(dtype)


def _plain_self(s):
    c, dt = s["case"], s["q"].dtype
    nq, nk = s["most_q"], s["most_k"]
    len_q = s["cu_q"][1:] - s["cu_q"][:-1]
    len_k = s["cu_k"][1:] - s["cu_k"][:-1] if s["len_k"] is None else s["len_k"]
    q, in_q = _padded(s["q"], s["cu_q"][:-1], len_q, nq)
    k, in_k = _padded(s["k"], s["cu_k"][:-1], len_k, nk)
    v, _ = _padded(s["v"], s["cu_k"][:-1], len_k, nk)
    # distances of a document: (len_k - len_q + i) - j
    first = (len_k - len_q).long()
    dist = first[:, None, None] + torch.arange(nq, device="cuda")[:, None] - torch.arange(nk, device="cuda")
    far = nq + nk
    by_distance = s["bias"].float()[_bucket(torch.arange(-far, far + 1, device="cuda"), c)].T       # [H, 2 far + 1]
    scale = 1.0 / math.sqrt(c["head_dim"])
    a = q @ k.transpose(2, 3) * scale + by_distance[:, dist + far].transpose(0, 1)
    seen = in_q[:, :, None] & in_k[:, None, :]
    if c["causal"]:
        seen = seen & (dist >= 0)
    a = torch.where(seen[:, None], a, -torch.inf)
    top = a.amax(3, keepdim=True).clamp(min=-1e30)
    p = torch.exp(a - top)
    del a
    total = p.sum(3, keepdim=True)
    lse = top + torch.log(total)
    p = p / total.clamp(min=1e-30)
    o = p @ v
    out = {"o": _packed(o, in_q, dt), "lse": lse[..., 0].transpose(0, 1)[:, in_q]}
    if not c["backward"]:
        return out
    do, _ = _padded(s["do"], s["cu_q"][:-1], len_q, nq)
    out["dv"] = _packed(p.transpose(2, 3) @ do, in_k, dt)
    ds = p * (do @ v.transpose(2, 3) - (do * o).sum(3, keepdim=True))
    del p
    out["dq"] = _packed(ds @ k * scale, in_q, dt)
    out["dk"] = _packed(ds.transpose(2, 3) @ q * scale, in_k, dt)
    # the diagonals of dS: keys turned round and rows sheared by one column each, so that column x holds the
    # distance first + x - (nk - 1)
    wide = torch.nn.functional.pad(ds.flip(3), (0, nq)).flatten(2)[..., :-nq].unflatten(2, (nq, nk + nq - 1))
    at = first[:, None] + torch.arange(nk + nq - 1, device="cuda") - (nk - 1)
    one = (_bucket(at, c)[:, :, None] == torch.arange(c["buckets"], device="cuda")).float()
    out["dbias"] = (wide.sum(2) @ one).sum(0).T.to(dt)
    return out


# ---- one pass: the library's calls ----------------------------------------------------------------
def _own(s):
    import paper_2407_08330_b200 as P
    c = s["case"]
    if c["kind"] == "drop":
        return {"y": P.hdt_dropout(s["x"], c["p"], s["rng"], site=s["site"], residual=s["residual"])}
    if c["kind"] == "norm" and not c["backward"]:
        y, h, mean, rstd = P.hdt_layer_norm_fwd(s["x"], s["weight"], s["bias"], residual=s["residual"], p=c["p"], rng=s["rng"], site=s["site"])
        return {"y": y, "h": h, "mean": mean, "rstd": rstd}
    if c["kind"] == "norm":
        dx, dres, dw, db = P.hdt_layer_norm_bwd(s["d_y"], s["h"], s["mean"], s["rstd"], s["weight"], d_h=s["d_h"], p=c["p"], rng=s["rng"], site=s["site"])
        return {"dx": dx, "dresidual": dres, "dweight": dw, "dbias": db}
    a = (s["cu_q"], s["cu_k"], s["q"], s["k"], s["v"])
    how = dict(bias=s["bias"], max_distance=c["max_distance"], causal=c["causal"], seqlens_k=s["len_k"])
    o, lse = P.hdt_self_attn_fwd(*a, **how)
    if not c["backward"]:
        return {"o": o, "lse": lse}
    dq, dk, dv, dbias = P.hdt_self_attn_bwd(*a, o, lse, s["do"], **how)
    return {"o": o, "lse": lse, "dv": dv, "dq": dq, "dk": dk, "dbias": dbias}


def run(s):
    if own:
        return _own(s)
    c = s["case"]
    if c["kind"] == "self":
        return _plain_self(s)
    if c["kind"] == "drop":
        return _plain_drop(s)
    return _plain_norm_bwd(s) if c["backward"] else _plain_norm_fwd(s)


# ---- what a pass cannot do without ----------------------------------------------------------------
def work(case):
    esz = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "drop":
        n = case["rows"] * case["cols"]
        return {"bytes": n * esz * (3 if case["residual"] else 2), "flops": n * 2}
    if case["kind"] == "norm":
        n, wsz = case["rows"] * case["cols"], 2 if case["w_dtype"] == "bf16" else 4
        changed = case["residual"] or case["p"] > 0          # h is another tensor than x
        if case["backward"]:
            # dy, h (and dh) in, the residual's gradient (and, with dropout, that of x) out
            return {"bytes": n * esz * (3 + case["residual"] + (case["p"] > 0)) + 8 * case["rows"] + 3 * case["cols"] * wsz, "flops": 14 * n}
        return {"bytes": n * esz * (2 + case["residual"] + changed) + 8 * case["rows"] + 2 * case["cols"] * wsz, "flops": 9 * n}
    n_q, n_k, _ = (x.astype(np.int64) for x in _lengths(case))
    H, d = case["heads"], case["head_dim"]
    # pairs of a document: row i of n_q sees n_k - n_q + i + 1 keys, or all
    pairs = int((n_q * (n_k - n_q) + n_q * (n_q + 1) // 2).sum()) if case["causal"] else int((n_q * n_k).sum())
    row, Tq, Tk = H * d * esz, int(n_q.sum()), int(n_k.sum())
    byt = 2 * Tq * row + 2 * Tk * row + 4 * H * Tq + case["buckets"] * H * esz
    if case["backward"]:      # q, k, v, o, do, lse, bias in; dq, dk, dv, dbias out
        byt += 4 * Tq * row + 4 * Tk * row + 4 * H * Tq + 2 * case["buckets"] * H * esz
    return {"bytes": byt, "flops": (14 if case["backward"] else 4) * d * pairs * H}


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _exact_keep(s, rows, cols):
    t = int(math.floor(65536 * s["case"]["p"] + 0.5))
    seed, offset = (int(x) for x in s["rng"].tolist())
    nb = (cols + 7) // 8
    m32 = np.uint64(0xFFFFFFFF)
    ctr = np.empty((4, rows, nb), np.uint64)
    ctr[0], ctr[1], ctr[2], ctr[3] = np.arange(nb)[None, :], np.arange(rows)[:, None], s["site"], offset & 0xFFFFFFFF
    key = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * ctr[0], np.uint64(0xCD9E8D57) * ctr[2]
        ctr = np.stack(((p1 >> np.uint64(32)) ^ ctr[1] ^ np.uint64(key[0]), p1 & m32, (p0 >> np.uint64(32)) ^ ctr[3] ^ np.uint64(key[1]), p0 & m32))
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = np.ascontiguousarray(ctr.transpose(1, 2, 0).astype("<u4")).view("<u2").reshape(rows, nb * 8)[:, :cols]
    keep = torch.from_numpy(halves >= t).cuda()
    return keep.double() * 65536 / (65536 - t)


def _exact_borders(n, far):
    """First distance of every bucket of one direction: integer arithmetic alone."""
    e = n // 2
    first = list(range(e + 1))
    for k in range(1, n - e):       # the smallest d with (d / e)^(n - e) >= (far / e)^k
        d = first[-1]
        while d ** (n - e) * e ** k < far ** k * e ** (n - e):
            d += 1
        first.append(d)
    return torch.tensor(first, device="cuda")


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] != "self":
        D = _exact_keep(s, case["rows"], case["cols"]) if case["p"] > 0 else 1.0
        if case["kind"] == "drop" or not case["backward"]:
            h = s["x"].double() * D
            if s["residual"] is not None:
                h += s["residual"].double()
            if case["kind"] == "drop":
                return {"y": h}
            var, mean = torch.var_mean(h, 1, correction=0)
            rstd = 1 / torch.sqrt(var + 1e-5)
            return {"y": torch.addcmul(s["bias"].double(), (h - mean[:, None]) * rstd[:, None], s["weight"].double()), "h": h, "mean": mean, "rstd": rstd}
        dy, r = s["d_y"].double(), s["rstd"].double()[:, None]
        u = s["h"].double().sub_(s["mean"].double()[:, None]).mul_(r)
        dw, db = torch.einsum("rc,rc->c", dy, u), dy.sum(0)
        g = dy * s["weight"].double()
        proj = torch.einsum("rc,rc->r", g, u) / case["cols"]
        dres = r * (g - g.sum(1, keepdim=True) / case["cols"] - u * proj[:, None])
        if s["d_h"] is not None:
            dres += s["d_h"].double()
        return {"dx": dres * D, "dresidual": dres, "dweight": dw, "dbias": db}
    n_q, n_k, room = _lengths(case)
    if case["heads"] * int((n_q.astype(np.int64) * n_k).sum()) > 4_000_000_000:
        return None
    H, d, n = case["heads"], case["head_dim"], case["buckets"]
    one_way = n if case["causal"] else n // 2
    borders = _exact_borders(one_way, case["max_distance"])
    t64 = {x: s[x].double() for x in ("q", "k", "v", "bias")}
    out = {"o": torch.zeros_like(t64["q"]), "lse": torch.zeros(H, int(n_q.sum()), dtype=torch.float64, device="cuda")}
    if case["backward"]:
        out |= {"dv": torch.zeros_like(t64["v"]), "dq": torch.zeros_like(t64["q"]), "dk": torch.zeros_like(t64["k"]), "dbias": torch.zeros_like(t64["bias"])}
    for b in range(case["batch"]):
        q0, k0 = int(n_q[:b].sum()), int(room[:b].sum())
        rq, rk = slice(q0, q0 + int(n_q[b])), slice(k0, k0 + int(n_k[b]))
        if n_q[b] == 0:
            continue
        delta = torch.arange(int(n_k[b] - n_q[b]), int(n_k[b]), device="cuda")[:, None] - torch.arange(int(n_k[b]), device="cuda")[None, :]
        bucket = torch.searchsorted(borders, delta.clamp(min=0) if case["causal"] else delta.abs(), right=True) - 1
        if not case["causal"]:
            bucket += one_way * (delta < 0)
        for h in range(H):
            q, k, v = t64["q"][rq, h], t64["k"][rk, h], t64["v"][rk, h]
            a = q @ k.T / math.sqrt(d) + t64["bias"][:, h][bucket]
            if case["causal"]:
                a.masked_fill_(delta < 0, -math.inf)
            lse = torch.logsumexp(a, 1)
            p = (a - lse[:, None]).exp_()
            o = p @ v
            out["o"][rq, h], out["lse"][h, rq] = o, lse
            if case["backward"]:
                do = s["do"][rq, h].double()
                ds = p * (do @ v.T - (do * o).sum(1, keepdim=True))
                out["dv"][rk, h], out["dq"][rq, h], out["dk"][rk, h] = p.T @ do, ds @ k / math.sqrt(d), ds.T @ q / math.sqrt(d)
                out["dbias"][:, h] += torch.bincount(bucket.flatten(), ds.flatten(), minlength=n)
    return out
