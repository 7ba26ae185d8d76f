"""Self-attention with a relative position bias on the GPU against the 64-bit definition.

Bounds (u = half a step of the type relative to the value; e = what fp32 adds, below).  bf16 calls round P, dS and every
result to 8 significant bits; delta comes from the rounded O:
  O      u |O| + (u + e) sum_j P |V|
  dV     u |dV| + (u + e) sum_i P |dO|
  delta  |dO| . (bound of O)                        =: D_i
  dQ     u |dQ| + scale sum_j [(u + e) |dS| + P (D_i + e |dO| |V|)] |K|, dK alike
  dBias  u |dBias| + sum over the bucket's pairs of [e |dS| + P (D_i + e |dO| |V|)]
fp32 calls: the same with u = 0 for P and dS.  e: a logit is a sum of d products, off by at most d 2^-24 sum |q k| scale; with
the bias, the maximum and the LSE, each a rounding of a number of at most A = max |a| + |LSE|, P is off by a factor of
(d + 16) 2^-24 (L + A) with L = the largest sum of |q k| scale; sums over up to n pairs and the exponential's own error
(2 units in the last place) add (n + d + 16) 2^-24.  LSE: (d + 16) 2^-24 (L + A) + n 2^-24."""
import numpy as np
import pytest
import torch

from oracle import self_oracle as S

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f32": torch.float32}
NAMES = ("o", "lse", "dq", "dk", "dv", "dbias")


def f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    """Packed documents: rows of q, keys, unused rows behind each document's keys, rows behind the last document."""

    def __init__(self, lens_q, lens_k, H, d, dtype, causal=True, buckets=32, far=128, bias=True, room=0, behind=0, seed=0, scale=0.0, fill=float("nan")):
        g = np.random.default_rng(seed + 7 * sum(lens_k) + H + d)
        self.lq, self.lk, self.H, self.d, self.causal, self.far, self.dtype = lens_q, lens_k, H, d, causal, far, dtype
        self.scale, self.scale_arg = (scale or d ** -0.5), scale
        self.cq = np.concatenate([[0], np.cumsum(lens_q)]).astype(np.int32)
        self.ck = np.concatenate([[0], np.cumsum(np.array(lens_k) + room)]).astype(np.int32)
        self.Tq, self.Tk = int(self.cq[-1]) + behind, int(self.ck[-1]) + behind
        t = lambda *s: torch.from_numpy(g.normal(size=s)).to(T[dtype]).cuda()
        self.q, self.k, self.v, self.do = t(self.Tq, H, d), t(self.Tk, H, d), t(self.Tk, H, d), t(self.Tq, H, d)
        self.bias = t(buckets, H) if bias else None
        self.len_k = torch.from_numpy(np.array(lens_k, np.int32)).cuda() if room else None
        for b, n in enumerate(lens_k):      # rows that belong to nothing
            for x in (self.k, self.v):
                x[self.ck[b] + n:self.ck[b + 1]] = fill
        for x in (self.q, self.do):
            x[self.cq[-1]:] = fill
        for x in (self.k, self.v):
            x[self.ck[-1]:] = fill
        self.cu = [torch.from_numpy(x).cuda() for x in (self.cq, self.ck)]

    def args(self):
        return (*self.cu, self.q, self.k, self.v), dict(bias=self.bias, max_distance=self.far, causal=self.causal, seqlens_k=self.len_k, softmax_scale=self.scale_arg)

    def run(self, backward=True, mark=-7.0):
        import paper_2407_08330_b200 as P
        a, kw = self.args()
        o, lse = torch.full_like(self.q, mark), torch.full((self.H, self.Tq), mark, device="cuda")
        P.hdt_self_attn_fwd(*a, out=o, lse=lse, **kw)
        got = dict(o=o, lse=lse)
        if backward:
            dq, dk, dv = torch.full_like(self.q, mark), torch.full_like(self.k, mark), torch.full_like(self.k, mark)
            got["dbias"] = P.hdt_self_attn_bwd(*a, o, lse, self.do, dq=dq, dk=dk, dv=dv, **kw)[3]
            got.update(dq=dq, dk=dk, dv=dv)
        P.hdt_device_status()
        return got

    def check(self, got):
        u = torch.finfo(T[self.dtype]).eps / 2
        up = u if self.dtype == "bf16" else 0.0
        backward = "dq" in got
        want_db = bound_db = 0.0
        worst = 0.0

        def near(name, x, y, bound, where):
            fin = np.isfinite(y)
            assert np.array_equal(np.isfinite(x), fin) and np.array_equal(x[~fin], y[~fin]), f"{name} {where}: other non-finite values"
            over = np.abs(x[fin] - y[fin]) - bound[fin] * 1.01 - 1e-30
            assert (over <= 0).all(), f"{name} {where}: off by {np.abs(x[fin] - y[fin]).max():.3e}, worst excess {over.max():.3e}"

        used_q, used_k = np.zeros(self.Tq, bool), np.zeros(self.Tk, bool)
        with np.errstate(invalid="ignore"):
            for b in range(len(self.lq)):
                rq, rk = slice(self.cq[b], self.cq[b + 1]), slice(self.ck[b], self.ck[b] + self.lk[b])
                used_q[rq], used_k[rk] = True, True
                if self.lq[b] == 0 and self.lk[b] == 0:
                    continue
                q, k, v, do = f64(self.q[rq]), f64(self.k[rk]), f64(self.v[rk]), f64(self.do[rq])
                bias = None if self.bias is None else f64(self.bias)
                w = S.document(q, k, v, bias, self.far, self.causal, self.scale, do)
                p = w["p"]
                n, f = max(self.lq[b], self.lk[b]), 2.0 ** -24
                L = self.scale * np.einsum("ihc,jhc->hij", np.abs(q), np.abs(k)).max(initial=0)
                A = 2 * L + 2 * (0 if bias is None else np.abs(np.where(np.isfinite(bias), np.clip(bias, -32768, 32768), 0)).max()) + np.log(n + 1.0)
                e = f * ((self.d + 16) * (L + A) + n + self.d + 16)
                where = f"document {b} of {self.lq[b]} rows, {self.lk[b]} keys"
                near("lse", f64(got["lse"][:, rq]), w["lse"], np.full(w["lse"].shape, e), where)
                bo = u * np.abs(w["o"]) + (up + e) * np.einsum("hij,jhc->ihc", p, np.abs(v))
                near("o", f64(got["o"][rq]), w["o"], bo, where)
                if not backward:
                    continue
                ds = np.abs(w["ds"])
                x = p * (np.einsum("ihc,ihc->hi", np.abs(do), bo)[..., None] + e * np.einsum("ihc,jhc->hij", np.abs(do), np.abs(v)))
                y = (up + e) * ds + x
                near("dv", f64(got["dv"][rk]), w["dv"], u * np.abs(w["dv"]) + (up + e) * np.einsum("hij,ihc->jhc", p, np.abs(do)), where)
                near("dq", f64(got["dq"][rq]), w["dq"], u * np.abs(w["dq"]) + self.scale * np.einsum("hij,jhc->ihc", y, np.abs(k)), where)
                near("dk", f64(got["dk"][rk]), w["dk"], u * np.abs(w["dk"]) + self.scale * np.einsum("hij,ihc->jhc", y, np.abs(q)), where)
                if bias is not None:
                    want_db = want_db + w["dbias"]
                    z = np.zeros_like(bias)
                    np.add.at(z, w["bucket"].reshape(-1), (e * ds + x).transpose(1, 2, 0).reshape(-1, self.H))
                    bound_db = bound_db + z
        if backward and self.bias is not None:
            near("dbias", f64(got["dbias"]), want_db, u * np.abs(want_db) + bound_db, "")
        # rows of no document are left as they were
        for name, used in (("o", used_q), ("dq", used_q), ("dk", used_k), ("dv", used_k)):
            if name in got and (~used).any():
                assert (got[name][torch.from_numpy(~used).cuda()] == -7).all(), name
        assert (got["lse"][:, torch.from_numpy(~used_q).cuda()] == -7).all()


LENGTHS = [([5], [5]), ([127], [127]), ([128], [128]), ([129], [129]), ([300], [300]), ([64, 65, 1, 130, 700], [64, 65, 1, 130, 700]),
           ([70, 30, 400], [100, 380, 400]), ([70, 100, 0, 50, 7], [40, 100, 9, 0, 300]), ([257, 2], [600, 260])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda x: "x".join(map(str, x[0])))
def test_parity(dtype, d, causal, lens):
    c = Case(*lens, 2, d, dtype, causal)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("buckets, far", [(2, 2), (4, 3), (3, 40), (16, 64), (64, 500), (128, 32768), (64, 100)])
@pytest.mark.parametrize("causal", [True, False])
def test_buckets(dtype, buckets, far, causal):
    if not causal and (buckets < 4 or buckets % 2):
        pytest.skip("at least two buckets a direction")
    c = Case([400, 33], [400, 290], 3, 64, dtype, causal, buckets, far)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_unused_rows_of_a_cache_and_behind_the_last_document(dtype, causal):
    c = Case([200, 3, 131], [300, 77, 131], 2, 64, dtype, causal, room=19, behind=40)
    c.check(c.run())
    c = Case([200, 3, 131], [300, 77, 131], 2, 128, dtype, causal, room=19, behind=40, fill=float("inf"))
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, H", [(64, 12), (128, 5), (64, 1)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [([1], [1]), ([1] * 6, [1, 2000, 64, 65, 700, 0]), ([4, 1, 2, 7, 0], [30, 500, 100, 90, 5]), ([8, 0, 0], [900, 4, 0]),
                                  ([1] * 40, list(range(40))), ([2] * 3, [1, 1, 129]), ([0, 0, 3], [5, 0, 2]),
                                  ([1, 0, 3, 0, 0, 1, 7] * 12, [9, 4, 300, 0, 8, 0, 70] * 12), ([1] * 1100, [i % 9 for i in range(1099)] + [900])], ids=lambda x: "x".join(map(str, x[0][:5])))
def test_decoding(dtype, d, H, causal, lens):
    for room in (0, 5):
        c = Case(*lens, H, d, dtype, causal, room=room, behind=3)
        c.check(c.run(backward=False))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_bias_and_a_scale_of_the_caller(dtype):
    c = Case([300, 20], [300, 90], 2, 64, dtype, True, bias=False, scale=0.05)
    c.check(c.run())
    c = Case([1, 1], [300, 90], 2, 64, dtype, True, bias=False, scale=0.05)
    c.check(c.run(backward=False))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[260, 90], [1, 1]])
def test_shut_buckets(dtype, rows):
    """-inf for the near buckets (rows that see nothing else are empty), and the type's lowest value, which counts as -32768."""
    c = Case(rows, [260, 90], 2, 64, dtype, True)
    c.bias[:5] = -torch.inf
    c.bias[20:] = -torch.inf
    c.check(c.run(backward=rows[0] > 1))
    c.bias[:] = torch.randn_like(c.bias)
    c.bias[:3] = -32768.0
    want = c.run(backward=False)
    c.check(want)
    c.bias[:3] = torch.finfo(T[dtype]).min
    got = c.run(backward=False)
    assert all(torch.equal(got[n], want[n]) for n in got)


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows", [[700, 400], [1, 1]])
def test_shut_far_bucket(dtype, d, causal, rows):
    """Nothing but the last bucket shut (whole tiles of it come first), or all but the first, or everything: logits that large that a
    weight of a shut key would not stay finite."""
    c = Case(rows, [700, 400], 3, d, dtype, causal, scale=20 / d ** 0.5)
    c.bias[:, 0] = -torch.inf
    c.bias[1 if causal else 31, 1] = -torch.inf
    c.bias[15:16, 1] = -torch.inf
    c.bias[31:, 1] = -torch.inf
    c.bias[1:, 2] = -torch.inf
    c.check(c.run(backward=rows[0] > 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_other_documents_stay_out_of_non_finite_ones(dtype, d):
    c = Case([140, 150, 60], [140, 150, 60], 2, d, dtype, True)
    clean = c.run()
    bad = slice(140, 290)
    for x in (c.q, c.k, c.v, c.do):
        x[bad] = float("nan")
    got = c.run()
    for n in ("o", "dq", "dk", "dv"):
        assert torch.equal(got[n][:140], clean[n][:140]) and torch.equal(got[n][290:], clean[n][290:]), n
    assert torch.equal(got["lse"][:, :140], clean["lse"][:, :140]) and torch.equal(got["lse"][:, 290:], clean["lse"][:, 290:])


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_repeated_calls_give_the_same_bits(dtype, d):
    c = Case([500, 333, 129], [500, 333, 129], 6, d, dtype, True, 64, 300)
    first = c.run()
    for _ in range(3):
        again = c.run()
        assert all(torch.equal(first[n], again[n]) for n in NAMES)
    s = Case([1] * 4, [900, 50, 3, 1200], 6, d, dtype)
    first = s.run(backward=False)
    assert all(torch.equal(first[n], s.run(backward=False)[n]) for n in first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_many_short_documents(dtype, d, causal):
    """Several units of one tile, and of none, in a row for every CTA."""
    lens = [(37 * i) % 150 for i in range(90)]
    keys = [0 if i % 11 == 0 else n + (i % 3) * 40 for i, n in enumerate(lens)]
    c = Case(lens, keys, 5, d, dtype, causal)
    c.check(c.run())


@pytest.mark.parametrize("rows", [[300, 129], [1, 1]])
def test_captured_and_replayed_with_other_lengths(rows):
    """Offsets are read on the device: one captured call serves whatever lengths the arrays hold at the replay."""
    import paper_2407_08330_b200 as P
    c = Case(rows, [300, 129], 4, 64, "bf16", room=8)
    a, kw = c.args()
    step = rows[0] == 1
    o, lse = torch.empty_like(c.q), torch.empty((4, c.Tq), device="cuda")

    def call():
        P.hdt_self_attn_fwd(*a, out=o, lse=lse, **kw)
        return (o, lse) if step else (o, lse) + P.hdt_self_attn_bwd(*a, o, lse, c.do, **kw)
    for x in (c.k, c.v):
        x[:] = torch.randn(x.shape, device="cuda").bfloat16()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            out = call()
    torch.cuda.synchronize()
    for lens in ((300, 129), (301, 137), (308, 130)):
        c.len_k.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        # (rows of k and v behind the lengths are not written: compared where they are)
        used = torch.zeros(c.Tk, dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            used[int(c.ck[b]):int(c.ck[b]) + n] = True
        for x, y in zip(kept, want):
            assert torch.equal(x[used], y[used]) if x.shape[0] == c.Tk else torch.equal(x, y)


def test_two_streams_at_once():
    import paper_2407_08330_b200 as P
    cs = [Case([700, 200], [700, 200], 8, 64, "bf16", seed=s) for s in (1, 2)]
    want = [c.run() for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    got = [None, None]
    for _ in range(3):
        for i, (c, s) in enumerate(zip(cs, streams)):
            a, kw = c.args()
            with torch.cuda.stream(s):
                o, lse = P.hdt_self_attn_fwd(*a, **kw)
                got[i] = (o, lse) + P.hdt_self_attn_bwd(*a, o, lse, c.do, **kw)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w[n]) for x, n in zip(g, NAMES))


def test_caches_beyond_2_31_elements():
    """Keys at rows whose element number does not fit 32 bits, by a step of decoding and by a chunk of rows."""
    import paper_2407_08330_b200 as P
    H, d, Tk = 12, 64, 2_800_000
    assert Tk * H * d > 2 ** 31
    k, v = (torch.empty(Tk, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu_k = torch.tensor([0, 5, Tk - 1000, Tk], dtype=torch.int32, device="cuda")
    lens = torch.tensor([5, 7, 900], dtype=torch.int32, device="cuda")
    for x in (k, v):
        for a, n in ((0, 5), (5, 7), (Tk - 1000, 900)):
            x[a:a + n] = torch.randn(n, H, d, device="cuda").bfloat16()
    bias = torch.randn(32, H, device="cuda").bfloat16()
    for rows in ([1, 1, 1], [0, 0, 200]):
        cu_q = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")
        q = torch.randn(sum(rows), H, d, device="cuda").bfloat16()
        o, lse = P.hdt_self_attn_fwd(cu_q, cu_k, q, k, v, bias=bias, seqlens_k=lens)
        small_k, small_v = (torch.cat([x[:12], x[Tk - 1000:Tk - 100]]) for x in (k, v))
        cu_s = torch.tensor([0, 5, 12, 912], dtype=torch.int32, device="cuda")
        o2, lse2 = P.hdt_self_attn_fwd(cu_q, cu_s, q, small_k, small_v, bias=bias)
        assert (lse - lse2).abs().max() < 1e-4 and (o.float() - o2.float()).abs().max() <= 2 ** -8 * 4
        P.hdt_device_status()


def test_no_rows_no_keys():
    import paper_2407_08330_b200 as P
    z = lambda n: torch.zeros(n, 2, 64, device="cuda").bfloat16()
    cu = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    bias = torch.randn(32, 2, device="cuda").bfloat16()
    o, lse = P.hdt_self_attn_fwd(cu(0, 9, 9), cu(0, 0, 0), z(9), z(0), z(0), bias=bias)
    assert not o.any() and torch.isneginf(lse).all()
    dq, dk, dv, db = P.hdt_self_attn_bwd(cu(0, 9, 9), cu(0, 0, 0), z(9), z(0), z(0), o, lse, z(9), bias=bias)
    assert not dq.any() and not db.any()
    o, lse = P.hdt_self_attn_fwd(cu(0, 0), cu(0, 7), z(0), z(7), z(7), bias=bias)
    dk, dv = z(7) + 1, z(7) + 1
    _, dk, dv, db = P.hdt_self_attn_bwd(cu(0, 0), cu(0, 7), z(0), z(7), z(7), o, lse, z(0), bias=bias, dk=dk, dv=dv)
    assert not dk.any() and not dv.any() and not db.any()
    assert P.hdt_self_attn_bwd(cu(0), cu(0), z(0), z(0), z(0), o, lse, z(0), bias=bias)[3].abs().max() == 0
    P.hdt_device_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_outside_the_tensors_are_clamped(dtype):
    """The kernels clamp what they read (see `document` there): no row outside is touched, the valid documents are right."""
    c = Case([60, 70], [60, 70], 2, 64, dtype, behind=30)
    want = c.run()
    for x in (c.q, c.k, c.v, c.do):
        x[130:] = 0.5
    valid = c.cu
    tail = lambda *x: [torch.cat([t, torch.tensor([n if n < 1000 else total + n for n in x], dtype=torch.int32, device="cuda")]) for t, total in zip(valid, (c.Tq, c.Tk))]
    c.cu = tail(1999, 3000, -5)                   # a document to the end of the tensors and two empty ones
    got = c.run()
    for n in ("o", "dq", "dk", "dv"):
        assert torch.equal(got[n][:130], want[n][:130]), n
    c.cu = tail(1999, -5, 1999)                   # the last one is the whole tensor again: rows of several documents are anyone's
    got = c.run()
    assert all(t.isfinite().all() for t in got.values())


def test_binding_refusals():
    import paper_2407_08330_b200 as P
    c = Case([20], [20], 2, 64, "bf16")
    a, kw = c.args()
    o, lse = P.hdt_self_attn_fwd(*a, **kw)
    f = P.hdt_self_attn_fwd
    for call in (lambda: f(c.cu[0].long(), *a[1:], **kw), lambda: f(c.cu[0][:1], *a[1:], **kw), lambda: f(*a[:2], c.q.float(), c.k, c.v, **kw),
                 lambda: f(*a[:2], c.q, c.k[:5], c.v, **kw), lambda: f(*a, **{**kw, "bias": c.bias.float()}), lambda: f(*a, **{**kw, "bias": c.bias[:, :1]}),
                 lambda: f(*a, **{**kw, "bias": c.bias.t().contiguous().t()}), lambda: f(*a, **{**kw, "max_distance": 3}), lambda: f(*a[:2], c.q.cpu(), c.k, c.v, **kw),
                 lambda: f(*a, **kw, lse=lse.t()), lambda: f(*a, **kw, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")),
                 lambda: f(*a[:2], *(x[..., ::2] for x in a[2:]), **kw), lambda: P.hdt_self_attn_bwd(*a, o, lse, c.do.float(), **kw)):
        with pytest.raises(P.HdtError):
            call()
