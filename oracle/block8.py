"""Oracle of a decoder block that runs in 8 bits (test infrastructure; numpy, imports nothing from the GPU package):
quantised linear, queries and keys normalised and rotated, appends to a paged cache of codes, attention over it.
Grid arithmetic (steps, quotients, codes) is float32 with one rounding an operation, as the definitions say; everything
else is float64."""
from __future__ import annotations

import numpy as np

F32 = np.float32
FLOOR = F32(1e-5)


def row_codes(x, bits, factor=None):
    """(codes int8 [n, c], steps float32 [n])."""
    xt = np.asarray(x, F32)
    if factor is not None:
        xt = xt * np.asarray(factor, F32)[None, :]
    top = F32(2 ** (bits - 1) - 1)
    step = np.maximum(np.abs(xt).max(axis=1), FLOOR) / top
    codes = np.clip(np.rint(xt / step[:, None]), -top - F32(1), top)
    return codes.astype(np.int8), step.astype(F32)


def linear_i8(x, bits, w_codes, w_steps, factor=None):
    codes, step = row_codes(x, bits, factor)
    sums = codes.astype(np.float64) @ w_codes.astype(np.float64).T          # exact: below 2^53
    return sums * np.asarray(w_steps, np.float64)[None, :] * step.astype(np.float64)[:, None]


def qk_norm_rope(x, head_dim, pos, inv_freq, w=None, eps=1e-6, norm=True, interleaved=False):
    """One of the two matrices, [n, heads * head_dim] -> float64."""
    n = x.shape[0]
    u = np.asarray(x, np.float64).reshape(n, -1, head_dim).copy()
    if norm:
        u /= np.sqrt((u * u).mean(axis=2, keepdims=True) + np.float64(F32(eps)))
        if w is not None:
            u *= np.asarray(w, np.float64)
    half = len(inv_freq)
    out = u.copy()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = pos.astype(np.float64) * float(inv_freq[i])
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[:, :, a] = u[:, :, a] * c - u[:, :, b] * s
        out[:, :, b] = u[:, :, b] * c + u[:, :, a] * s
    return out.reshape(n, -1)


def sequence(cu, lens, s, n_tok, page, max_pages, max_len):
    """(first row, new rows, position of the first new row, tokens in reach)."""
    r0 = min(max(int(cu[s]), 0), n_tok)
    r1 = min(max(int(cu[s + 1]), r0), n_tok)
    n = max(int(lens[s]), 0)
    return r0, r1 - r0, n - (r1 - r0), min(n, max_len, max_pages * page)


def kv_append(x, codes, steps, cu, lens, table, max_len, transposed):
    """New rows x [n_tok, heads * dh] into codes [pages, heads, page, dh] (transposed: [pages, heads, dh, page]) and steps, in
    place."""
    n_pages, heads = steps.shape
    page, dh = codes.shape[2:] if not transposed else codes.shape[:1:-1]
    x = np.asarray(x, F32)
    for s in range(len(lens)):
        r0, n_new, first, n = sequence(cu, lens, s, x.shape[0], page, table.shape[1], max_len)
        begin = max(first, 0)
        for p in range(begin // page, (n - 1) // page + 1 if n > begin else 0):
            pid = int(table[s, p])
            if not 0 <= pid < n_pages:
                continue
            lo, hi = max(begin - p * page, 0), min(n - p * page, page)
            rows = r0 + p * page - first + np.arange(lo, hi)
            for h in range(heads):
                v = x[rows, h * dh:(h + 1) * dh]
                fin = np.where(np.isfinite(v), np.abs(v), F32(0))
                step = np.maximum(fin.max(), FLOOR) / F32(127)
                page_codes = codes[pid, h].T if transposed else codes[pid, h]       # views: [page, dh]
                if lo > 0:
                    was = steps[pid, h]
                    step = was if was > step else step
                    if was != step:
                        page_codes[:lo] = np.rint(page_codes[:lo].astype(F32) * (was / step)).astype(np.int8)
                with np.errstate(invalid="ignore"):
                    q = np.clip(np.rint(v / step), -127, 127)
                page_codes[lo:hi] = np.where(np.isnan(v), 0, q).astype(np.int8)
                steps[pid, h] = step


def kv_attention(q, heads, kc, ks, vc, vs, cu, lens, table, max_len, scale=None):
    """(out, mag, sens) float64 [n_tok, heads * dh]: mag = sum_j p_j |v_j| and sens [n_tok, heads] = the largest of
    scale * sum_d |q_d| |k_jd|, which bound what roundings can do.  Rows of no sequence are NaN."""
    n_pages, kv, page, dh = kc.shape
    n_tok, group = q.shape[0], heads // kv
    scale = 1.0 / np.sqrt(dh) if not scale else float(F32(scale))
    out = np.full((n_tok, heads * dh), np.nan)
    mag, sens = out.copy(), np.zeros((n_tok, heads))
    q = np.asarray(q, np.float64)
    for s in range(len(lens)):
        r0, n_new, first, n = sequence(cu, lens, s, n_tok, page, table.shape[1], max_len)
        ids = [int(i) for i in table[s, :-(-n // page)]] if n > 0 else []
        there = np.repeat(np.array([0 <= i < n_pages for i in ids], bool), page)[:n]
        ids = [i if 0 <= i < n_pages else 0 for i in ids]
        for h in range(kv):
            if ids:
                k = np.concatenate([kc[i, h].astype(np.float64) * float(ks[i, h]) for i in ids])[:n]
                v = np.concatenate([vc[i, h].T.astype(np.float64) * float(vs[i, h]) for i in ids])[:n]
                k[~there], v[~there] = 0.0, 0.0            # (their steps may be anything)
            for g in range(group):
                c = slice((h * group + g) * dh, (h * group + g + 1) * dh)
                for r in range(n_new):
                    m = min(first + r + 1, n)
                    see = there[:m] if m > 0 else np.zeros(0, bool)
                    if not see.any():
                        out[r0 + r, c] = mag[r0 + r, c] = 0.0
                        continue
                    kk, vv = k[:m][see], v[:m][see]
                    z = scale * (kk @ q[r0 + r, c])
                    p = np.exp(z - z.max())
                    p /= p.sum()
                    out[r0 + r, c] = p @ vv
                    mag[r0 + r, c] = p @ np.abs(vv)
                    sens[r0 + r, h * group + g] = abs(scale) * (np.abs(kk) @ np.abs(q[r0 + r, c])).max()
    return out, mag, sens
