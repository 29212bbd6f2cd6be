"""Plain forms of the paged 4-bit KV cache and of rotary positions for the tests: the quantizer step by
step in IEEE fp32 (its definition), everything else in 64 bits."""
import numpy as np

from kv8_reference import random_batch, sees  # noqa: F401  (for the tests)

STEP = np.float32(1) / np.float32(7)


def bf16_bits(x):
    """float32 -> bfloat16 bits, nearest even (no NaN)."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def bf16_value(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32)


def quant(x):
    """(codes int8, scale bits) of float16 rows [..., D]."""
    with np.errstate(all="ignore"):
        x = x.astype(np.float32)
        bits = bf16_bits(np.fmax.reduce(np.abs(x), axis=-1, initial=np.float32(0)) * STEP)
        s = bf16_value(bits)[..., None]
        c = np.rint(x / np.where(s > 0, s, np.float32(1)))
        return np.where((s > 0) & ~np.isnan(c), c, 0).astype(np.int8), bits


def pack(c):
    c = c.astype(np.uint8) & 15
    return c[..., 0::2] | (c[..., 1::2] << 4)


def unpack(b):
    c = np.stack((b & 15, b >> 4), axis=-1).reshape(*b.shape[:-1], -1).astype(np.int8)
    return np.where(c > 7, c - 16, c)


def values(codes, bits):
    """What packed codes and scale bits stand for: float16."""
    with np.errstate(all="ignore"):
        return (bf16_value(bits)[..., None] * unpack(codes).astype(np.float32)).astype(np.float16)


def places(cu, lens, table, P):
    """(row, page, slot) of each row that has a place in the cache."""
    for s in range(len(lens)):
        n, L = int(cu[s + 1] - cu[s]), int(lens[s])
        for i in range(max(n - L, 0), n):
            p = L - n + i
            yield int(cu[s]) + i, int(table[s, p // P]), p % P


def append(codes, bits, rows, cu, lens, table):
    c, b = quant(rows)
    for r, page, at in places(cu, lens, table, codes.shape[2]):
        codes[page, :, at], bits[page, :, at] = pack(c[r]), b[r]


def read(codes, bits, out, cu, lens, table):
    """Writes the cached values of the batch's rows into out."""
    for r, page, at in places(cu, lens, table, codes.shape[2]):
        out[r] = values(codes[page, :, at], bits[page, :, at])


def attend(cache, q, cu, lens, table, scale, window=0, sinks=0):
    """(out, tolerance), both float64 [tokens, heads, dim].  The tolerance follows the roundings that the
    operator declares: fp32 logits (dot products of D products, relative 2^-24 a step), weights
    rounded to binary16 (2^-11 relative; below its normal range 2^-25 of a unit of which the largest weight, or the
    largest weight times V scale, is at least 2^7), fp32 sums, one rounding to binary16."""
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
        vis = sees(L - n + np.arange(n), L, window, sinks) & held[None]
        for h in range(H):
            K, V = (values(c[pages, h], b[pages, h]).reshape(-1, D)[:L].astype(np.float64) for c, b in ((kc, ks), (vc, vs)))
            C = np.abs(unpack(vc[pages, h])).reshape(-1, D)[:L].astype(np.float64)
            sv = bf16_value(vs[pages, h]).reshape(-1)[:L].astype(np.float64)
            x = q[cu[s]:cu[s] + n, h * g:(h + 1) * g].astype(np.float64).transpose(1, 0, 2)   # [g, n, D]
            a = np.where(vis, x @ K.T * scale, -np.inf)
            mag = np.abs(x) @ np.abs(K).T * abs(scale)
            m = a.max(axis=2, keepdims=True)
            w = np.exp(a - np.where(np.isfinite(m), m, 0))
            l = w.sum(axis=2, keepdims=True)
            w = np.divide(w, l, out=np.zeros_like(w), where=l > 0)
            o = w @ V
            # an error d of a logit moves its weight by d relative, above and below the line
            logit = (D + 16) * 2.0 ** -23 * np.where(vis, mag, 0).max(axis=2, keepdims=True)
            rel = 2.0 ** -11 + 2 * logit + (L / 16 + 64) * 2.0 ** -23
            cut = 2.0 ** -32 * (w.max(axis=2, keepdims=True) * (vis @ np.abs(V)) +
                                (w * sv).max(axis=2, keepdims=True) * (vis @ C))
            t = rel * (w @ np.abs(V)) + cut + 2.0 ** -11 * np.abs(o) + 2.0 ** -24
            out[cu[s]:cu[s] + n, h * g:(h + 1) * g] = o.transpose(1, 0, 2)
            tol[cu[s]:cu[s] + n, h * g:(h + 1) * g] = t.transpose(1, 0, 2)
    return out, tol


def random_cache(rng, blocks, H, P, D):
    """Full-range codes (packed) and scale bits that differ between tokens by several binades."""
    c = [pack(rng.integers(-7, 8, (blocks, H, P, D)).astype(np.int8)) for _ in range(2)]
    b = [bf16_bits((0.3 * 2.0 ** rng.uniform(-3, 2, (blocks, H, P))).astype(np.float32)) for _ in range(2)]
    return [c[0], b[0], c[1], b[1]]


def frequencies(r, base=10000.0, scaling="none", factor=1.0, trained_len=0.0, low=1.0, high=4.0):
    i = np.arange(r // 2)
    if scaling == "ntk":
        base = base * factor ** (r / (r - 2))
    f = base ** (-2.0 * i / r)
    if scaling == "linear":
        return f / factor
    turns = trained_len * f / (2 * np.pi)
    if scaling == "wavelength":
        keep = np.clip((turns - low) / (high - low), 0, 1)
    elif scaling == "ramp":
        d = [r * np.log(trained_len / (2 * np.pi * t)) / (2 * np.log(base)) for t in (high, low)]
        a, b = max(np.floor(d[0]), 0), min(np.ceil(d[1]), r - 1)
        keep = 1 - np.clip((i - a) / max(b - a, 0.001), 0, 1)
    else:
        keep = np.ones(len(i))
    return keep * f + (1 - keep) * f / factor


def rotate(x, pos, freq, interleaved, amplitude=1.0):
    """(out, tolerance) float64 of rotary positions on float16 rows [tokens, heads, dim]; rows at negative
    positions stay.  Angles off by half a unit in the last place of an fp32 number of half turns below one
    (pi 2^-25), cos and sin by another 2 units of 2^-24, an amplitude, two products and a sum rounded: together
    under 2^-21 of (|x1| + |x2|); one rounding to binary16."""
    r = 2 * len(freq)
    y = x.astype(np.float64)
    tol = np.zeros_like(y)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    th = np.asarray(pos, np.float64)[:, None, None] * freq
    c, s = np.cos(th) * amplitude, np.sin(th) * amplitude
    u, v = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    tol[..., a] = tol[..., b] = 2.0 ** -21 * abs(amplitude) * (np.abs(u) + np.abs(v)) + 2.0 ** -25
    tol[..., :r] += 2.0 ** -11 * np.abs(y[..., :r])
    stay = np.asarray(pos) < 0
    y[stay], tol[stay] = x[stay].astype(np.float64), 0
    return y, tol
