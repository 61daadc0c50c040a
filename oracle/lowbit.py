"""Oracle of the block's other calls in low bits (test infrastructure; numpy, imports nothing from the GPU package): residual, norm
and codes; products of codes with an epilogue; rotation by positions on several axes; the cache in 4 bits, attention over it.
Grid arithmetic (steps, quotients, codes) has the types that the definitions name, one rounding an operation; everything else
is float64."""
from __future__ import annotations

import math

import numpy as np

from oracle.block8 import FLOOR, sequence
from oracle.tlq_oracle import round_to_bf16

F32 = np.float32
GROUP = 32
SHIFT = [4 * (e // 2) + 16 * (e % 2) for e in range(8)]


def round16(x, bf16):
    """float32 -> the nearest value of the type, as float32."""
    x = np.asarray(x, F32)
    return np.asarray(round_to_bf16(x), F32) if bf16 else x.astype(np.float16).astype(F32)


def add_norm_codes(h, z, w, eps, bits, bf16):
    """(h + z rounded, codes int8, steps float32) of rows of 16-bit values."""
    h = np.asarray(h, F32) if z is None else round16(np.asarray(h, F32) + np.asarray(z, F32), bf16)
    mean = np.array([math.fsum(np.asarray(r, np.float64) ** 2) for r in h]) / h.shape[1]
    with np.errstate(divide="ignore"):
        r = (1.0 / np.sqrt(mean + np.float64(F32(eps)))).astype(F32)
    u = h * r[:, None]
    if w is not None:
        u = u * np.asarray(w, F32)[None, :]
    top = F32(2 ** (bits - 1) - 1)
    step = np.maximum(np.abs(u).max(axis=1), FLOOR) / top
    return h, np.clip(np.rint(u / step[:, None]), -top - F32(1), top).astype(np.int8), step.astype(F32)


def act(v, kind):
    """0 none, 1 SiLU, 2 GELU in its tanh form, 3 GELU."""
    v = np.asarray(v, np.float64)
    with np.errstate(over="ignore"):
        if kind == 1:
            return v / (1.0 + np.exp(-v))
        if kind == 2:
            return v / (1.0 + np.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    if kind == 3:
        return v * 0.5 * np.vectorize(math.erfc)(-v / math.sqrt(2.0))
    return v


def linear_codes(codes, steps, w_codes, w_steps, bias, kind, r, mul):
    """(y, the product in front of the bias, v = product + bias, act(v)) in float64."""
    p = (codes.astype(np.float64) @ w_codes.astype(np.float64).T) * np.asarray(w_steps, np.float64)[None, :] * np.asarray(steps, np.float64)[:, None]
    v = p if bias is None else p + np.asarray(bias, np.float64)[None, :]
    a = act(v, kind)
    y = a if r is None else a * r if mul else a + r
    return y, p, v, a


def norm_rope_axes(x, head_dim, pos, axis, inv_freq, w=None, eps=1e-6, norm=True, interleaved=False):
    """One of the two matrices, [n, heads * head_dim] -> float64; pos [axes, n]."""
    n = x.shape[0]
    u = np.asarray(x, np.float64).reshape(n, -1, head_dim).copy()
    if norm:
        u /= np.sqrt((u * u).mean(axis=2, keepdims=True) + np.float64(F32(eps)))
        if w is not None:
            u *= np.asarray(w, np.float64)
    half, out = len(inv_freq), u.copy()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        turn = np.exp(1j * pos[min(max(int(axis[i]), 0), len(pos) - 1)].astype(np.float64) * float(inv_freq[i]))[:, None]
        z = (u[:, :, a] + 1j * u[:, :, b]) * turn
        out[:, :, a], out[:, :, b] = z.real, z.imag
    return out.reshape(n, -1)


# ------------------------------------------------------------------ the cache in 4 bits
def pack(codes):
    """codes [..., c] in -8..7 -> int32 words [..., c / 8]."""
    n = (np.asarray(codes, np.int64) + 8).reshape(*codes.shape[:-1], -1, 8)
    w = sum(n[..., e] << SHIFT[e] for e in range(8))
    return w.astype(np.uint32).view(np.int32)


def unpack(words):
    w = np.ascontiguousarray(words).view(np.uint32)
    return np.stack([(w >> np.uint32(s)) & np.uint32(15) for s in SHIFT], -1).reshape(*words.shape[:-1], -1).astype(np.int64) - 8


def quantise(x):
    """Rows [n, c] -> (codes int8 [n, c], steps float16 [n, c / 32])."""
    x = np.asarray(x, F32).reshape(x.shape[0], -1, GROUP)
    most = np.where(np.isfinite(x), np.abs(x), F32(0)).max(axis=2)
    with np.errstate(over="ignore", invalid="ignore"):
        step = np.minimum(np.asarray(round_to_bf16(np.maximum(most, FLOOR) / F32(7)), F32).astype(np.float16), np.float16(9344.0))
        q = np.clip(np.rint(x / step.astype(F32)[..., None]), -7, 7)
    return np.where(np.isnan(x), 0, q).astype(np.int8).reshape(x.shape[0], -1), step


def kv4_append(x, codes, steps, cu, lens, table, max_len, transposed, max_new=None):
    """New rows x [n_tok, heads * dh] into codes [pages, heads, page, dh] (transposed: [.., dh, page]) and steps [.., page, dh / 32]
    ([.., dh / 32, page]), in place."""
    n_pages, heads = codes.shape[:2]
    page, dh = codes.shape[2:] if not transposed else codes.shape[:1:-1]
    q, st = quantise(x)
    for s in range(len(lens)):
        r0, n_new, first, n = sequence(cu, lens, s, x.shape[0], page, table.shape[1], max_len)
        if max_new is not None:
            n = min(n, first + min(n_new, max_new))
        for t in range(max(first, 0), n):
            pid = int(table[s, t // page])
            if not 0 <= pid < n_pages:
                continue
            c, v = q[r0 + t - first].reshape(heads, dh), st[r0 + t - first].reshape(heads, dh // GROUP)
            if transposed:
                codes[pid, :, :, t % page], steps[pid, :, :, t % page] = c, v
            else:
                codes[pid, :, t % page], steps[pid, :, t % page] = c, v


def values(codes, steps, transposed):
    """Pools of float64 values [pages, heads, page, dh] (or [.., dh, page])."""
    s = np.asarray(steps, np.float64)
    return codes * np.repeat(s, GROUP, axis=2 if transposed else 3)


def kv4_read(codes, steps, cu, lens, table, n_tok, max_len, transposed):
    """float64 [n_tok, heads * dh]; rows of no sequence are NaN."""
    n_pages, heads = codes.shape[:2]
    page, dh = codes.shape[2:] if not transposed else codes.shape[:1:-1]
    out = np.full((n_tok, heads * dh), np.nan)
    for s in range(len(lens)):
        r0, n_new, first, n = sequence(cu, lens, s, n_tok, page, table.shape[1], max_len)
        for r in range(n_new):
            t = first + r
            pid = int(table[s, t // page]) if 0 <= t < n else -1
            out[r0 + r] = 0.0
            if 0 <= pid < n_pages:
                c, v = (codes[pid, :, :, t % page], steps[pid, :, :, t % page]) if transposed else (codes[pid, :, t % page], steps[pid, :, t % page])
                out[r0 + r] = (c * np.repeat(v.astype(np.float64), GROUP, axis=1)).ravel()
    return out


def attention(q, heads, kpool, vpool, cu, lens, table, max_len, scale=None):
    """Over pools of values [pages, kv, page, dh] and [pages, kv, dh, page] -> (out, mag, sens) float64: mag = sum_j p_j |v_j| and
    sens [n_tok, heads] = the largest of |scale| * sum_d |q_d| |k_jd|, which bound what roundings can do.  Rows of no sequence are NaN."""
    n_pages, kv, page, dh = kpool.shape
    n_tok, group = q.shape[0], heads // kv
    scale = 1.0 / math.sqrt(dh) if not scale else float(F32(scale))
    out = np.full((n_tok, heads * dh), np.nan)
    mag, sens = out.copy(), np.zeros((n_tok, heads))
    q = np.asarray(q, np.float64)
    for s in range(len(lens)):
        r0, n_new, first, n = sequence(cu, lens, s, n_tok, page, table.shape[1], max_len)
        n = max(n, 0)
        ids = np.array(table[s, :-(-n // page)], np.int64)
        there = np.repeat((ids >= 0) & (ids < n_pages), page)[:n]
        ids = np.where((ids >= 0) & (ids < n_pages), ids, 0)
        for h in range(kv):
            k = kpool[ids, h].reshape(-1, dh)[:n][there]
            v = vpool[ids, h].transpose(0, 2, 1).reshape(-1, dh)[:n][there]
            where = np.flatnonzero(there)
            for r in range(n_new):
                m = int(np.searchsorted(where, first + r, side="right"))
                cols = slice(h * group * dh, (h + 1) * group * dh)
                if m == 0:
                    out[r0 + r, cols] = mag[r0 + r, cols] = 0.0
                    continue
                x = q[r0 + r, cols].reshape(group, dh)
                with np.errstate(invalid="ignore"):
                    z = scale * (x @ k[:m].T)
                    p = np.exp(z - z.max(axis=1, keepdims=True))
                    p /= p.sum(axis=1, keepdims=True)
                    out[r0 + r, cols] = (p @ v[:m]).ravel()
                    mag[r0 + r, cols] = (p @ np.abs(v[:m])).ravel()
                    sens[r0 + r, h * group:(h + 1) * group] = abs(scale) * (np.abs(x) @ np.abs(k[:m]).T).max(axis=1)
    return out, mag, sens
