"""What a serving step computes around its linears (oracle; test infrastructure):
RMS norm with 8-bit codes, the 8-bit paged KV cache, attention over it, and log
probabilities of tokens.  Codes and cache scales are pinned bit for bit; all
else is evaluated in float64 from the definitions.
"""

import numpy as np

__all__ = ["rms_norm_quant_ref", "e4m3_values", "e4m3_encode", "kv8_scale", "kv8_append_ref", "kv8_values",
           "kv8_attention_ref", "token_logprobs_ref", "PAGE"]

PAGE = 64


def rms_norm_quant_ref(x, weight, eps, residual=None):
    """fp16 [M, K] -> (codes int8, scales float64 [M], h fp16)."""
    h = np.asarray(x, np.float16)
    if residual is not None:
        h = (h.astype(np.float32) + np.asarray(residual, np.float16).astype(np.float32)).astype(np.float16)
    t = h.astype(np.float32) * np.asarray(weight, np.float16).astype(np.float32)      # exact
    s = (np.abs(t).max(1) / np.float32(127)).astype(np.float32)
    q = t / np.where(s > 0, s, np.float32(1))[:, None]
    codes = np.where(s[:, None] > 0, np.rint(q), 0).astype(np.int8)
    h64 = h.astype(np.float64)
    with np.errstate(divide="ignore"):
        r = 1 / np.sqrt((h64 ** 2).mean(1) + eps)
    return codes, np.where(s > 0, s * np.where(s > 0, r, 0), 0.0), h


def e4m3_values():
    """The 256 values of OCP e4m3 (0x7F and 0xFF are NaN, there is no infinity)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e.astype(float) - 7))
    v[(c & 0x7F) == 0x7F] = np.nan
    return np.where(c >= 128, -v, v)


def e4m3_encode(x):
    """Codes of float64 values |x| <= 448, nearest, ties to the even code."""
    x = np.asarray(x, np.float64)
    grid = e4m3_values()[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(grid, a, side="left"), 1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (c | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def kv8_scale(absmax):
    """The smallest 2^e with absmax <= 448 * 2^e, e >= -32."""
    e = -32
    while absmax > 448.0 * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


def kv8_append_ref(k, v, cu, lengths, table, cache):
    """New tokens [T, H, D] into copies of (k_pages u8 [P, H, 64, D], v_pages u8 [P, H, D, 64], k_scales, v_scales)."""
    cache = [np.array(c) for c in cache]
    P, values = cache[0].shape[0], e4m3_values()
    for pages, scales, rows, turned in ((cache[0], cache[2], k, False), (cache[1], cache[3], v, True)):
        for b in range(len(lengths)):
            count = cu[b + 1] - cu[b]
            start = lengths[b] - count
            for blk in range(max(start, 0) // PAGE, (lengths[b] + PAGE - 1) // PAGE):
                lo, hi = max(start, 0, blk * PAGE), min(lengths[b], (blk + 1) * PAGE)
                if lo >= hi or blk >= table.shape[1] or not 0 <= table[b, blk] < P:
                    continue
                page = table[b, blk]
                for h in range(pages.shape[1]):
                    x = rows[cu[b] + lo - start:cu[b] + hi - start, h].astype(np.float64)
                    codes = pages[page, h].T if turned else pages[page, h]     # a view [64, D]
                    s = kv8_scale(np.abs(x).max())
                    first = lo - blk * PAGE
                    if first:
                        had = scales[page, h]
                        s = max(s, had)
                        if s > had:
                            codes[:first] = e4m3_encode(values[codes[:first]] * (float(had) / float(s)))
                    else:
                        codes[hi - blk * PAGE:] = 0
                    codes[first:hi - blk * PAGE] = e4m3_encode(x / float(s))
                    scales[page, h] = s
    return cache


def kv8_values(cache, pages, head):
    """float64 K and V [64 * len(pages), D] of one head."""
    values = e4m3_values()
    k = [values[cache[0][p, head]] * float(cache[2][p, head]) for p in pages]
    v = [values[cache[1][p, head]].T * float(cache[3][p, head]) for p in pages]
    return np.concatenate(k), np.concatenate(v)


def kv8_attention_ref(q, cu, lengths, table, cache, scale, window=0, sinks=0):
    """(out, lse, bounds) in float64: bounds of the rounding that the library's formula admits, for out and lse."""
    T, H, D = q.shape
    P, Hkv = cache[0].shape[:2]
    out, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    tol_out, tol_lse = np.zeros((T, H, D)), np.zeros((T, H))
    for b in range(len(lengths)):
        n, c = int(lengths[b]), int(cu[b + 1] - cu[b])
        blocks = min((n + PAGE - 1) // PAGE, table.shape[1])
        if c == 0 or n == 0 or blocks == 0:
            continue
        pages = [int(p) for p in table[b, :blocks]]
        held = np.repeat([0 <= p < P for p in pages], PAGE)
        j = np.arange(blocks * PAGE)
        for hk in range(Hkv):
            k, v = kv8_values(cache, [p if 0 <= p < P else 0 for p in pages], hk)
            for i in range(c):
                p = n - c + i
                see = held & (j <= p)
                if window:
                    see &= (j > p - window) | (j < sinks)
                if not see.any():
                    continue
                ks, vs = k[see], v[see]
                for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                    x = q[cu[b] + i, h].astype(np.float64)
                    s = scale * (ks @ x)
                    m = s.max()
                    w = np.exp(s - m)
                    out[cu[b] + i, h] = (w @ vs) / w.sum()
                    lse[cu[b] + i, h] = m + np.log(w.sum())
                    # Scores: D products and sums in fp32, two scale factors.
                    ds = (D + 16) * 2.0 ** -24 * abs(scale) * (np.abs(ks) @ np.abs(x)).max()
                    # The hardware's exponential, running rescales, n fp32 sums.
                    rel = 2 * ds + (len(s) + 64) * 2.0 ** -24 + 2.0 ** -20
                    # P to fp16: half an ulp, or half the smallest subnormal step.
                    mean = (w @ np.abs(vs)) / w.sum()
                    floor = 2.0 ** -25 * np.abs(vs).sum(0) / w.sum()
                    o = np.abs(out[cu[b] + i, h])
                    tol_out[cu[b] + i, h] = mean * (2.0 ** -12 + 2 * rel) + floor + o * 2.0 ** -11 + 2.0 ** -24
                    tol_lse[cu[b] + i, h] = rel + 2.0 ** -21 * (abs(m) + 1 + np.log(len(s)))
    return out, lse, tol_out, tol_lse


def token_logprobs_ref(logits, tokens, top=0):
    """(logprobs, entropy, top_logprobs, top_ids) in float64."""
    x = np.asarray(logits).astype(np.float64)
    M, V = x.shape
    lp, ent = np.zeros(M), np.zeros(M)
    tops, ids = np.full((M, top), -np.inf), np.zeros((M, top), np.int64)
    for r in range(M):
        order = np.lexsort((np.arange(V), -x[r]))[:top]
        ids[r] = order
        m = x[r].max()
        if m == -np.inf:
            lse = None
        else:
            lse = m + np.log(np.exp(x[r] - m).sum())
            y = x[r] - lse
            p = np.exp(y)
            ent[r] = -np.sum(p[p > 0] * y[p > 0])
            tops[r] = y[order]
        t = tokens[r]
        if t >= V:
            lp[r] = np.nan
        elif t >= 0:
            lp[r] = -np.inf if lse is None else x[r, t] - lse
    return lp, ent, tops, ids
