"""Plain 64-bit forms of the paged operators (test infrastructure), with the
error bounds of the library's arithmetic beside them."""
import math

import numpy as np

EPS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # half a step, relative


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_length=0.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        keep = np.clip((f * original_length / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        return f * keep + f / factor * (1 - keep), 1.0 + 0.1 * math.log(factor)
    return f, 1.0


def rotate(x, pos, layout, f, mag):
    """(x [rows, heads, dim] turned, bound of the fp32 arithmetic).  The bound:
    a cosine or sine is off by at most 4 roundings (reduced angle, two in the
    series, magnitude), each product and the final sum by one: 6 * 2^-24 of
    m (|a| + |b|)."""
    r = 2 * len(f)
    x = np.asarray(x, np.float64)
    t = np.asarray(pos, np.float64)[:, None, None] * f
    c, s = mag * np.cos(t), mag * np.sin(t)
    ia, ib = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = x[..., ia], x[..., ib]
    out, err = x.copy(), np.zeros_like(x)
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    err[..., ia] = err[..., ib] = 6 * 2.0 ** -24 * mag * (np.abs(a) + np.abs(b))
    return out, err


def attend(q, K, V, pos, kind, scale=None, softcap=0.0, window=0, slopes=None, own=None):
    """One user: q [c, H, D] at positions pos [c]; K and V [Hkv, n, D]; own:
    (k, v) [c, Hkv, D] or None (causal).  Returns (out, bound).

    Weights: a score is a sum of D fp32 products (D + 3 roundings of the sum of
    their magnitudes, in units of the scaled score), the cap's tanh is off by
    2^-21 of the cap, the bias by two roundings, the exponent's argument by one
    of its size and the exponential by 2^-22; in bf16 models each weight is
    rounded to bf16 (2^-8).  The same holds for the normaliser: twice.  Sums
    over n keys add n roundings; the result is rounded once."""
    c, H, D = q.shape
    Hkv, n, _ = K.shape
    scale = D ** -0.5 if scale is None else scale
    out, bound = np.zeros((c, H, D)), np.zeros((c, H, D))
    j = np.arange(n)
    pos = np.asarray(pos)
    seen = (j[None] <= pos[:, None]) if own is None else np.ones((c, n), bool)
    if window:
        seen &= j[None] > pos[:, None] - window
    for h in range(H):
        g = h // (H // Hkv)
        Kh, Vh, vis = K[g], V[g], seen
        z = q[:, h] @ Kh.T
        mag = np.abs(q[:, h]) @ np.abs(Kh).T
        away = (j[None] - pos[:, None]).astype(np.float64)
        if own is not None:
            z = np.concatenate([z, (q[:, h] * own[0][:, g]).sum(-1, keepdims=True)], 1)
            mag = np.concatenate([mag, np.abs(q[:, h] * own[0][:, g]).sum(-1, keepdims=True)], 1)
            away = np.concatenate([away, np.zeros((c, 1))], 1)
            vis = np.concatenate([seen, np.ones((c, 1), bool)], 1)
        z = z * scale
        delta = (D + 3) * 2.0 ** -24 * mag * scale
        if softcap:
            z = softcap * np.tanh(z / softcap)
            delta = delta + 2.0 ** -21 * softcap
        if slopes is not None:
            z = z + slopes[h] * away
            delta = delta + 2 * 2.0 ** -24 * (np.abs(slopes[h] * away) + np.abs(z))
        z = np.where(vis, z, -np.inf)
        top = z.max(1, keepdims=True)
        p = np.exp(z - top)
        rel = np.where(vis, delta + 2.0 ** -22 + 2.0 ** -23 * (np.abs(np.where(vis, z, 0.0)) + np.abs(top)), 0.0)
        rel = rel + (EPS["bf16"] if kind == "bf16" else 0.0) + n * 2.0 ** -24
        w = p / p.sum(1, keepdims=True)
        def weighted(x, of):
            y = x[:, :n] @ of(Vh)
            return y if own is None else y + x[:, n:] * of(own[1][:, g])

        out[:, h] = weighted(w, np.asarray)
        size = weighted(w, np.abs)
        worst = (w * rel).sum(1, keepdims=True)         # of the normaliser
        bound[:, h] = weighted(w * rel, np.abs) + worst * size
        bound[:, h] += EPS[kind] * (np.abs(out[:, h]) + bound[:, h])
    return out, bound


class Pages:
    """A pool of pages on the GPU with users' rows in shuffled pages; unused
    places and pages hold `fill`."""

    def __init__(self, rng, kind, rows, Hkv, D, page, layers=None, extra_pages=2, fill=None, spare_rows=0):
        import torch
        self.kind, self.page, self.rows = kind, page, np.asarray(rows, np.int32)
        need = [-(-(int(n) + spare_rows) // page) for n in rows]
        total = sum(need) + extra_pages
        order = rng.permutation(total).astype(np.int32)
        width = max(need + [1]) + 1
        self.tables = np.full((len(rows), width), order[0] if total else 0, np.int32)
        at = 0
        for u, k in enumerate(need):
            self.tables[u, :k] = order[at:at + k]
            at += k
        shape = (total, 2, Hkv, page, D)
        self.dt = torch.bfloat16 if kind == "bf16" else torch.float32
        lead = () if layers is None else (layers,)
        data = torch.full(lead + shape, float("nan") if fill is None else fill, dtype=self.dt)
        self.hist = []
        for u, n in enumerate(rows):
            kv = torch.from_numpy(rng.standard_normal((2, Hkv, int(n), D)).astype(np.float32)).to(self.dt)
            self.hist.append(kv.double().numpy())
            if layers is None:
                for p in range(int(n)):
                    data[self.tables[u, p // page], :, :, p % page] = kv[:, :, p]
        self.data = data.cuda()
        self.tables_d = torch.from_numpy(self.tables).cuda()

    def cache(self):
        from paper_2606_00422_amd import upr
        return upr.PagedCache(self.data, self.tables_d)


def offsets(counts, first=0):
    return (first + np.concatenate([[0], np.cumsum(counts)])).astype(np.int32)


def normal(rng, kind, *shape, scale=1.0):
    """(GPU tensor of the kind, its values in float64)."""
    import torch
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32))
    t = t.to(torch.bfloat16 if kind == "bf16" else torch.float32)
    return t.cuda(), t.double().numpy()
