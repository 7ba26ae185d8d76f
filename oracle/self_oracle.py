"""Plain definition in 64 bits of self-attention with a learned bias by relative position, and its gradients.  Bucket
borders by integer arithmetic."""
import functools

import numpy as np


@functools.lru_cache(maxsize=None)
def borders(n, max_distance):
    """Smallest distance of every bucket of one direction with n buckets."""
    e = n // 2
    out = list(range(e + 1))
    for k in range(1, n - e):      # (d / e)^(n - e) >= (max_distance / e)^k
        lo, hi = out[-1], max_distance
        while lo < hi:
            mid = (lo + hi) // 2
            if mid ** (n - e) * e ** k >= max_distance ** k * e ** (n - e):
                hi = mid
            else:
                lo = mid + 1
        out.append(lo)
    return out


def bucket(d, num_buckets, max_distance, causal):
    """Buckets of an integer array of distances (position of the query minus the key's)."""
    n = num_buckets if causal else num_buckets // 2
    one = lambda x: np.searchsorted(borders(n, max_distance), x, side="right") - 1
    return one(np.maximum(d, 0)) if causal else one(np.abs(d)) + np.where(d < 0, n, 0)


def document(q, k, v, bias, max_distance, causal, scale, do=None):
    """One document: q [nq, H, d], k, v [nk, H, d], bias [buckets, H] or None.  Returns a dict."""
    nq, H, _ = q.shape
    nk = k.shape[0]
    dist = (nk - nq + np.arange(nq))[:, None] - np.arange(nk)[None, :]
    a = np.einsum("ihc,jhc->hij", q, k) * scale
    if bias is not None:
        b = bucket(dist, bias.shape[0], max_distance, causal)
        a = a + bias[b].transpose(2, 0, 1)
    seen = dist >= 0 if causal else np.ones_like(dist, bool)
    a = np.where(seen[None], a, -np.inf)
    top = a.max(2, initial=-np.inf, keepdims=True)
    use = np.where(np.isfinite(top), top, 0.0)
    p = np.exp(a - use)
    total = p.sum(2, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (use + np.log(total))[..., 0]
    p = p / np.where(total > 0, total, 1.0)
    o = np.einsum("hij,jhc->ihc", p, v)
    out = dict(o=o, lse=lse, p=p)
    if do is None:
        return out
    dp = np.einsum("ihc,jhc->hij", do, v)
    ds = p * (dp - np.einsum("ihc,ihc->hi", do, o)[..., None])
    out.update(dq=np.einsum("hij,jhc->ihc", ds, k) * scale, dk=np.einsum("hij,ihc->jhc", ds, q) * scale, dv=np.einsum("hij,ihc->jhc", p, do), ds=ds, dp=dp)
    if bias is not None:
        db = np.zeros_like(bias)
        np.add.at(db, b.reshape(-1), ds.transpose(1, 2, 0).reshape(-1, H))
        out.update(dbias=db, bucket=b)
    return out
