"""Oracle: the attention block (TEST INFRASTRUCTURE ONLY), float64.

* :func:`projection`: an int4 group-64 projection with its unmerged adapter
  (§2 Quantization; §3.3 Recovery LoRA), and the magnitude of its sums.
* :func:`cache_row`, :func:`rotate`: a latent cache row and the rotation of
  neighbouring pairs.
* :func:`attend`: attention of one head over latent rows, expanded, and the
  bounds that roundings of its operands are held to.
* :class:`Pages`: reference counts of cache pages.
"""

import numpy as np

from . import quant

EPS = 1e-6
HALF = 2.0 ** -11        # largest relative rounding error of fp16
SINGLE = 2.0 ** -24      # of fp32
TINY = 2.0 ** -25        # half of fp16's smallest step
WEIGHT = TINY / 128      # the same of a softmax weight that is held times 2^7, the row's largest at 2^7 or more


def projection(qsz, lora, lora_scale, x):
    """(y, magnitude): y = W x + s B (A x) for rows ``x``, and the same with every term of the two sums
    that a row is made of (codes and zeros, adapter) taken absolutely."""
    q, s, z = qsz
    x = np.asarray(x, np.float64)
    codes = quant.unpack_nibbles(q)
    w = quant.dequantize_g64(codes, s, z)
    y = x @ w.T
    zero = np.repeat(np.abs(np.asarray(z, np.float64)), 64, axis=1)
    scaled = np.abs(quant.dequantize_g64(codes, s, np.zeros_like(z)))
    mag = np.abs(x) @ (scaled + zero).T
    if lora is not None:
        a, b = (np.asarray(v, np.float64) for v in lora)
        y = y + lora_scale * (x @ a.T) @ b.T
        mag = mag + abs(lora_scale) * (np.abs(x) @ np.abs(a).T) @ np.abs(b).T
    return y, mag


def projection_bound(y, mag, in_dim, rank, f16):
    """Sums of at most 64 products, in_dim / 64 groups (two terms each), rank more and 16 partial sums in fp32,
    each rounding at most SINGLE of the magnitude; 2^-21 of it for the group sums and A x held as two halves
    (22 bits of each); one rounding to fp16."""
    e = (64 + 2 * (in_dim // 64) + 2 * rank + 16) * SINGLE * mag + 2.0 ** -21 * mag
    return e + (HALF * np.abs(y) + TINY if f16 else 0.0)


def rotate(v, cos, sin):
    out = np.empty_like(v, dtype=np.float64)
    out[..., 0::2] = v[..., 0::2] * cos - v[..., 1::2] * sin
    out[..., 1::2] = v[..., 0::2] * sin + v[..., 1::2] * cos
    return out


def cache_row(kv, gamma, cos, sin):
    kv, gamma = np.asarray(kv, np.float64), np.asarray(gamma, np.float64)
    n = gamma.shape[0]
    c = kv[..., :n] / np.sqrt(np.mean(kv[..., :n] ** 2, -1, keepdims=True) + EPS) * gamma
    return np.concatenate([c, rotate(kv[..., n:], cos, sin)], -1)


def rope_table(max_pos, d_rope, base=10000.0):
    """fp32 [max_pos, d_rope / 2, 2] of (cos, sin), the angles in float64."""
    f = base ** (-np.arange(0, d_rope, 2) / d_rope)
    a = np.arange(max_pos)[:, None] * f
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def attend(q, rows, w_uk, w_uv, scale, seen=None):
    """Queries ``q [n, Dn + Dr]`` of one head over latent ``rows [L, Dc + Dr]``; row i sees the first seen[i].
    Returns (o [n, Dv], bound): the bound is what the roundings to fp16 may add up to, to first order, each at
    its largest: in the absorbed form q in the latent space, the weights and the weighted latents, in the
    expanded one the keys, the weights and the values, and the output in both; fp32 sums on top."""
    q, rows = np.asarray(q, np.float64), np.asarray(rows, np.float64)
    w_uk, w_uv = np.asarray(w_uk, np.float64), np.asarray(w_uv, np.float64)
    n, Dn, Dc = q.shape[0], w_uk.shape[0], w_uk.shape[1]
    if seen is None:
        seen = np.full(n, len(rows))
    out, bound = np.zeros((n, w_uv.shape[0])), np.zeros((n, w_uv.shape[0]))
    live = np.asarray(seen) > 0
    if not live.any() or not len(rows):
        return out, bound
    lat, rope = rows[:, :Dc], rows[:, Dc:]
    s = scale * ((q[:, :Dn] @ w_uk) @ lat.T + q[:, Dn:] @ rope.T)
    s[np.arange(len(rows))[None] >= np.asarray(seen)[:, None]] = -np.inf
    s, ql = s[live], q[live]
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    p /= p.sum(-1, keepdims=True)
    o = (p @ lat) @ w_uv.T
    # a score's error: every factor of its sums off by HALF (rounded q~ or keys) and fp32 sums of Dc + Dr terms
    unit = HALF + (Dc + Dn) * SINGLE
    absq = scale * unit * ((np.abs(ql[:, :Dn]) @ np.abs(w_uk)) @ np.abs(lat).T + np.abs(ql[:, Dn:]) @ np.abs(rope).T)
    absq = np.where(p > 0, absq, 0.0)
    ds = absq.max(-1, keepdims=True)                     # (softmax: |dp / p| <= 2 max |ds|)
    mag = (p @ np.abs(lat)) @ np.abs(w_uv).T
    rel = 2 * ds + 3 * HALF + (len(rows) + Dc) * SINGLE  # + weights, latents or values, the output
    far = ((p > 0) @ np.abs(lat)) @ np.abs(w_uv).T       # (p's largest is at most 1: each is off by WEIGHT at most)
    out[live], bound[live] = o, rel * mag + WEIGHT * far + TINY
    return out, bound


class Pages:
    """Reference counts, lowest free ids first."""

    def __init__(self, n, page_tokens):
        self.refs, self.page = [0] * n, page_tokens

    def free_ids(self):
        return [i for i, r in enumerate(self.refs) if r == 0]

    def alloc(self, n):
        ids = self.free_ids()[:n]
        if len(ids) < n:
            return None
        for i in ids:
            self.refs[i] = 1
        return ids

    def fork(self, pages, n_tokens):
        n = -(-n_tokens // self.page)
        full = n_tokens // self.page
        if n > full and not self.free_ids():
            return None
        for i in pages[:full]:
            self.refs[i] += 1
        if n == full:
            return list(pages[:full]), []
        new = self.alloc(1)[0]
        return list(pages[:full]) + [new], [(pages[full], new)]

    def free(self, pages):
        left = list(self.refs)
        for i in pages:
            if not 0 <= i < len(left) or left[i] < 1:
                return False
            left[i] -= 1
        self.refs = left
        return True

    def compact(self):
        n_live = sum(r > 0 for r in self.refs)
        holes = [i for i in range(n_live) if self.refs[i] == 0]
        late = [i for i in range(n_live, len(self.refs)) if self.refs[i] > 0]
        remap = [i if r > 0 else -1 for i, r in enumerate(self.refs)]
        for a, b in zip(late, holes):
            remap[a] = b
            self.refs[b], self.refs[a] = self.refs[a], 0
        return list(zip(late, holes)), remap
