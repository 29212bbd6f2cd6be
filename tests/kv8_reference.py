"""Plain forms of the residual norm and of the int8 paged KV cache for the tests: the quantizers
step by step in IEEE fp32 (their definition), everything else in 64 bits."""
import numpy as np

STEP = np.float32(1) / np.float32(127)


def norm_quant(x, residual, gamma, eps, bits):
    """(h float16, codes int, scales float64) of the fused residual norm."""
    with np.errstate(all="ignore"):
        h = x if residual is None else (x.astype(np.float32) + residual.astype(np.float32)).astype(np.float16)
        p = h.astype(np.float32)
        if gamma is not None:
            p = p * gamma.astype(np.float32)          # exact: 11 + 11 bits
        step = np.float32(1) / np.float32(2 ** (bits - 1) - 1)
        s = np.fmax.reduce(np.abs(p), axis=1, initial=np.float32(0)) * step
        c = np.rint(p / np.where(s > 0, s, np.float32(1))[:, None])
        c = np.where(np.isnan(c), 0, c).astype(np.int64)
        rms = np.sqrt(np.mean(h.astype(np.float64) ** 2, axis=1) + eps)
        return h, c, s.astype(np.float64) / rms


def quant(x, s):
    with np.errstate(all="ignore"):
        c = np.rint(x.astype(np.float32) / np.where(s > 0, s, np.float32(1)))
        return np.where((s > 0) & ~np.isnan(c), c, 0).astype(np.int8)


def append(codes, scales, rows, cu, lens, table):
    """Writes `rows` (float16 [tokens, heads, dim]) into codes / scales, page by page."""
    P = codes.shape[2]
    for s in range(len(lens)):
        n, L = int(cu[s + 1] - cu[s]), int(lens[s])
        start = L - n
        first = max(start, 0)
        if n == 0 or L == 0:
            continue
        for page in range(first // P, (L - 1) // P + 1):
            b = table[s, page]
            lo, hi = max(first, page * P), min(L, (page + 1) * P)
            x = rows[cu[s] + lo - start:cu[s] + hi - start].astype(np.float32)          # [t, heads, dim]
            lo, hi = lo - page * P, hi - page * P
            with np.errstate(all="ignore"):
                s0 = scales[b].copy() if lo > 0 else np.zeros_like(scales[b])
                s1 = np.fmax(s0, np.fmax.reduce(np.abs(x), axis=(0, 2), initial=np.float32(0)) * STEP)
                for h in np.nonzero(s1 > s0)[0]:
                    codes[b, h, :lo] = quant(codes[b, h, :lo].astype(np.float32) * s0[h], s1[h])
            codes[b, :, lo:hi] = quant(x, s1[None, :, None]).transpose(1, 0, 2)
            scales[b] = s1


def sees(pos, L, window, sinks):
    j = np.arange(L)[None, :]
    p = np.asarray(pos)[:, None]
    v = j <= p
    if window:
        v = v & ((j > p - window) | (j < sinks))
    return v


def attend(cache, q, cu, lens, table, scale, window=0, sinks=0):
    """(out, tolerance), both float64 [tokens, heads, dim].  The tolerance follows the roundings
    that the operator declares: fp32 logits (dot products of D exact products, relative
    2^-24 a step), weights rounded to binary16 (2^-11 relative, 2^-25 of the row's largest
    below its normal range), fp32 sums, one rounding to binary16 at the end."""
    kc, ks, vc, vs = cache
    T, Hq, D = q.shape
    H, P = kc.shape[1], kc.shape[2]
    g = Hq // H
    out, tol = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    for s in range(len(lens)):
        n, L = int(cu[s + 1] - cu[s]), int(lens[s])
        if n == 0 or L == 0:
            continue
        pages = table[s, :-(-L // P)]
        held = np.repeat(pages >= 0, P)[:L]
        pages = np.maximum(pages, 0)
        pos = L - n + np.arange(n)
        vis = sees(pos, L, window, sinks) & held[None]
        for h in range(H):
            K = kc[pages, h].reshape(-1, D)[:L].astype(np.float64)
            V = vc[pages, h].reshape(-1, D)[:L].astype(np.float64)
            sk = np.repeat(ks[pages, h].astype(np.float64), P)[:L]
            sv = np.repeat(vs[pages, h].astype(np.float64), P)[:L]
            for e in range(h * g, (h + 1) * g):
                x = q[cu[s]:cu[s] + n, e].astype(np.float64)
                a = (x @ K.T) * sk * scale
                mag = (np.abs(x) @ np.abs(K).T) * sk * abs(scale)
                a = np.where(vis, a, -np.inf)
                m = a.max(axis=1, keepdims=True)
                w = np.exp(a - np.where(np.isfinite(m), m, 0))
                l = w.sum(axis=1, keepdims=True)
                w = np.divide(w, l, out=np.zeros_like(w), where=l > 0)
                ws = w * sv
                o = ws @ V
                # an error d of a logit moves its weight by d relative, above and below the line
                logit = (D + 16) * 2.0 ** -23 * np.where(vis, mag, 0).max(axis=1, keepdims=True)
                rel = 2.0 ** -11 + 2 * logit + (L / 16 + 64) * 2.0 ** -23
                cut = 2.0 ** -25 * ws.max(axis=1, keepdims=True, initial=0) * (vis @ np.abs(V))
                t = rel * (ws @ np.abs(V)) + cut + 2.0 ** -11 * np.abs(o) + 2.0 ** -24
                out[cu[s]:cu[s] + n, e], tol[cu[s]:cu[s] + n, e] = o, t
    return out, tol


def random_cache(rng, blocks, H, P, D):
    """Full-range codes and scales that differ between pages by several binades."""
    c = [rng.integers(-127, 128, (blocks, H, P, D)).astype(np.int8) for _ in range(2)]
    s = [(0.02 * 2.0 ** rng.uniform(-3, 3, (blocks, H))).astype(np.float32) for _ in range(2)]
    return [c[0], s[0], c[1], s[1]]


def random_batch(rng, ns, lens, P, blocks=None, spare=2):
    """cu, lens, block table (pages in random order, -1 where a sequence needs none), pages."""
    need = [-(-l // P) for l in lens]
    blocks = blocks or sum(need) + spare
    order = rng.permutation(blocks)
    table = np.full((len(lens), max(1, max(need, default=1))), -1, dtype=np.int32)
    at = 0
    for s, k in enumerate(need):
        table[s, :k] = order[at:at + k]
        at += k
    return np.concatenate([[0], np.cumsum(ns)]).astype(np.int32), np.asarray(lens, dtype=np.int32), table, blocks
