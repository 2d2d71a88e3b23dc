"""A decoder's operators from their definitions, in NumPy: products in 8-bit integers, appending to a paged cache with the rotation by positions, and
attention over it.  64 bits throughout, but for the codes of 8-bit integers, whose definition names the 32-bit operations that lead to them
(quantize_rows, append_int8); sequence by sequence and head by head."""
import numpy as np

F = np.float32


def quantize_rows(x):
    """x fp16 [M][K] -> codes int8, scales fp32: s = max|x| * (1 / 127), q = rint(x * (1 / s)), all in fp32; a row that is not finite: NaN and zeros."""
    x = np.asarray(x).astype(F)
    s = np.abs(x).max(1) * (F(1) / F(127))
    fine = np.isfinite(s)
    with np.errstate(divide="ignore", invalid="ignore"):
        inv = np.where(fine & (s > 0), F(1) / s, F(0)).astype(F)
        q = np.rint(x * inv[:, None])
    return np.where(fine[:, None], q, 0).astype(np.int8), np.where(fine, s, np.nan).astype(F)


def gemm_i8(x, xs, w, ws, bias=None, res=None):
    """Before the activation.  (In 64-bit floats the sums of products of 8-bit integers are exact.)"""
    y = x.astype(np.float64) @ w.astype(np.float64).T * xs.astype(np.float64)[:, None] * ws.astype(np.float64)[None]
    y = y + (0 if bias is None else bias.astype(np.float64))
    return y + (0 if res is None else res.astype(np.float64))


def pair(dim, interleaved):
    """Indices of the pairs that are rotated: (a, b) of each."""
    return (np.arange(0, dim, 2), np.arange(1, dim, 2)) if interleaved else (np.arange(dim // 2), np.arange(dim // 2, dim))


def rotate(x, position, dim, base, interleaved):
    """x [heads][D] at one position, 64 bits."""
    y = np.asarray(x, np.float64).copy()
    if dim:
        a, b = pair(dim, interleaved)
        angle = position * float(base) ** (-2.0 * np.arange(dim // 2) / dim)
        y[:, a] = x[:, a] * np.cos(angle) - x[:, b] * np.sin(angle)
        y[:, b] = x[:, b] * np.cos(angle) + x[:, a] * np.sin(angle)
    return y


def rotate32(x, row, interleaved):
    """x fp32 [heads][D] with the table's row, every product and sum rounded to fp32."""
    y = x.copy()
    if row is not None:
        dim = len(row)
        a, b = pair(dim, interleaved)
        c, s = row[:dim // 2].astype(F), row[dim // 2:].astype(F)
        y[:, a] = x[:, a] * c - x[:, b] * s
        y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def places(q_start, kv_len, table, page_tokens, pages, max_q, max_kv, tokens):
    """(sequence, token, position, page or -1, row) of every token that is worked on."""
    for b in range(len(kv_len)):
        q0, q1 = (min(max(int(v), 0), tokens) for v in (q_start[b], q_start[b + 1]))
        n, total = max(q1 - q0, 0), min(max(int(kv_len[b]), 0), max_kv)
        for i in range(min(n, max_q)):
            p = total - n + i
            g = int(table[b][p // page_tokens]) if p >= 0 else -1
            yield b, q0 + i, p, g if 0 <= g < pages else -1, p % page_tokens


def append_int8(codes, scale, x, where, rope, interleaved):
    """codes int8 [pages][heads][P][D], scale fp32 [pages][heads], both changed; x fp16 [tokens][heads][D]; where: places(); rope: the table or None."""
    new = {}
    x = np.clip(np.nan_to_num(x.astype(F), nan=0.0), -65504, 65504)
    for _, t, p, g, row in where:
        if p >= 0 and g >= 0:
            new.setdefault(g, []).append((row, rotate32(x[t], None if rope is None else rope[p], interleaved)))
    for g, rows in new.items():
        first = min(r for r, _ in rows)
        top = np.max([np.abs(y).max(1) for _, y in rows], 0).astype(F)
        before = scale[g] if first else np.zeros_like(top)
        now = np.maximum(before, top * (F(1) / F(127))).astype(F)
        for h in range(len(now)):
            if first and now[h] > before[h]:
                codes[g, h, :first] = np.rint(codes[g, h, :first].astype(F) * (before[h] / now[h])).astype(np.int8)
            inv = F(1) / now[h] if now[h] > 0 else F(0)
            for r, y in rows:
                codes[g, h, r] = np.rint(y[h] * inv).astype(np.int8)
        scale[g] = now


def attention(q, k, v, position, scale, window, sinks, there=None):
    """One sequence and head: q [n][D] at `position` [n], k and v [keys][D] in 64 bits; there [keys]: keys that may be seen at all.  Returns the output, and
    the same sum with |v| (for bounds of the error), both zero where nothing is seen."""
    j = np.arange(len(k))
    at = position[:, None] - j[None]
    seen = at >= 0
    if window:
        seen &= (at < window) | (j[None] < sinks)
    if there is not None:
        seen &= there[None]
    k, v = np.where(seen.any(0)[:, None], k, 0), np.where(seen.any(0)[:, None], v, 0)
    s = np.where(seen, q @ k.T * scale, -np.inf)
    top = s.max(1, initial=-np.inf, keepdims=True)
    p = np.exp(s - np.where(top > -np.inf, top, 0))
    p /= np.maximum(p.sum(1, keepdims=True), 1e-300)
    return p @ v, p @ np.abs(v)
