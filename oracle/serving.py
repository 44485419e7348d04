"""CPU oracle for the batched serving operations: rows of several sequences
with paged key/value caches, and sampling.

TEST INFRASTRUCTURE ONLY: imported by the test suite, never by the library,
and sharing no code with the HIP path.  Float64, one row at a time, from the
plain definitions (the norm, rotation and softmax of oracle/decode.py):

  sequence b owns rows start[b] .. start[b+1]-1, the last of its seq_len[b]
  positions; position t lies in page table[b][t // page_size], slot
  t % page_size; pages are [num_pages][Hkv][page_size][d] arrays.
"""
import math

import numpy as np

from . import decode as D


def rows(start, seq_len):
    """(row, sequence, position) of every row that some sequence owns."""
    for b in range(len(seq_len)):
        n = int(start[b + 1]) - int(start[b])
        for i in range(n):
            yield int(start[b]) + i, b, int(seq_len[b]) - n + i


def place(table, b, t, page_size, num_pages):
    """(page, slot) of position t, or None where there is none."""
    if t < 0 or t // page_size >= table.shape[1]:
        return None
    page = int(table[b, t // page_size])
    return (page, t % page_size) if 0 <= page < num_pages else None


def turn(x, cos_sin_row):
    """Rotates the half-split pairs of x [..., d] by the angles whose cosines,
    then sines, are given."""
    half = x.shape[-1] // 2
    c, s = cos_sin_row[:half], cos_sin_row[half:]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def paged_append(qkv, q_w, k_w, cos_sin, k_pages, v_pages, table, start, seq_len, Hq, eps, q_out):
    """Returns (q_out, k_pages, v_pages) in float64, rows and slots that the
    call does not write as they were."""
    P, Hkv, ps, d = k_pages.shape
    q, kc, vc = (np.array(a, dtype=np.float64) for a in (q_out, k_pages, v_pages))
    for r, b, pos in rows(start, seq_len):
        if pos < 0 or pos >= cos_sin.shape[0] or pos >= table.shape[1] * ps:
            q[r] = 0
            continue
        x = np.asarray(qkv[r], dtype=np.float64).reshape(Hq + 2 * Hkv, d)
        cs = np.asarray(cos_sin[pos], dtype=np.float64)
        parts = []
        for y, w in ((x[:Hq], q_w), (x[Hq:Hq + Hkv], k_w)):
            parts.append(turn(y if w is None else D.rmsnorm(y, w, eps), cs))
        q[r] = parts[0]
        at = place(table, b, pos, ps, P)
        if at is not None:
            kc[at[0], :, at[1]] = parts[1]
            vc[at[0], :, at[1]] = x[Hq + Hkv:]
    return q, kc, vc


def paged_attention(q, k_pages, v_pages, table, start, seq_len, window, out):
    """Returns (out, weight, reach): the outputs (rows of no sequence as they
    were), the softmax weights' sum of |v| per output, and the largest
    sum |q_d k_d| / sqrt(d) per row and head: what rounding errors scale with."""
    P, Hkv, ps, d = k_pages.shape
    Hq = q.shape[1]
    R = Hq // Hkv
    out = np.array(out, dtype=np.float64)
    weight = np.zeros_like(out)
    reach = np.zeros(out.shape[:2])
    for r, b, pos in rows(start, seq_len):
        seen = [place(table, b, t, ps, P) for t in range(max(0, pos - window + 1) if window else 0, pos + 1)]
        seen = [s for s in seen if s is not None]
        out[r] = 0
        if not seen:
            continue
        pg, sl = (np.array(x) for x in zip(*seen))
        for g in range(Hkv):
            K, V = (c[pg, g, sl].astype(np.float64) for c in (k_pages, v_pages))
            for h in range(g * R, (g + 1) * R):
                x = q[r, h].astype(np.float64)
                s = K @ x / math.sqrt(d)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[r, h] = p @ V
                weight[r, h] = p @ np.abs(V)
                reach[r, h] = (np.abs(K) @ np.abs(x)).max() / math.sqrt(d)
    return out, weight, reach


def sample_row(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row, by walking the tokens in order."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    top = x[order[0]]
    if top == -np.inf:
        return -1, 0.0
    if not temperature > 0:
        return order[0], 1.0
    w = [1.0 if x[i] == top else math.exp((x[i] - top) / float(temperature)) for i in order]
    if 0 < top_k < len(w):
        w = w[:top_k]
    whole = math.fsum(w)
    n = len(w)
    if top_p < 1:
        run = 0.0
        for i, a in enumerate(w):
            run += a
            if run >= max(float(top_p), 0.0) * whole:
                n = min(n, i + 1)
                break
    if min_p > 0:
        n = min(n, sum(a >= min(float(min_p), 1.0) for a in w))
    while n > 1 and x[order[n - 1]] == -np.inf:  # never drawn
        n -= 1
    w = w[:n]
    kept = math.fsum(w)
    u = float(u) if u > 0 else 0.0
    run = 0.0
    for i, a in enumerate(w if u < 1 else []):  # (the sum of all may be rounded above `kept` before the last)
        run += a
        if run > u * kept:
            return order[i], a / kept
    return order[n - 1], w[-1] / kept


# ---------------------------------------------------------------------------
# caches of 8 bits: e4m3 codes, an e8m0 scale for each 16 positions of a head
# ---------------------------------------------------------------------------
BLOCK = 16
LOWEST, HIGHEST = 112, 134


def e4m3_values():
    """float64 [256]: the numbers that the codes stand for."""
    out = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = math.nan if c & 127 == 127 else math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
        out.append(-v if c & 128 else v)
    return np.array(out)


def e4m3(x):
    """Codes of float64 values: the nearest, of two the even one; saturated;
    0x7F where not finite."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0)
    v = e4m3_values()[:127]  # 0 .. 448, ascending
    i = np.clip(np.searchsorted(v, a, side="right") - 1, 0, 125)
    below, above = a - v[i], v[i + 1] - a
    c = np.where((above < below) | ((above == below) & (i % 2 == 1)), i + 1, i)
    c = np.where(np.signbit(x), c | 128, c)
    return np.where(np.isfinite(x), c, 127).astype(np.uint8)


def least_scale(a):
    """The least of 112..134 with a <= 448 * 2^(scale - 127), else 134."""
    for s in range(LOWEST, HIGHEST):
        if a <= math.ldexp(448.0, s - 127):
            return s
    return HIGHEST


def clamp_scale(s):
    return min(max(int(s), LOWEST), HIGHEST)


def cache_values(codes, scales):
    """float64 [P][Hkv][page_size][d] of codes and scales [P][Hkv][page_size / 16]."""
    s = np.repeat(np.clip(scales.astype(np.int64), LOWEST, HIGHEST) - 127, BLOCK, axis=2)
    return np.ldexp(e4m3_values()[codes], s[..., None])


def paged_append_e4m3(qkv, q_w, k_w, cos_sin, caches, table, start, seq_len, Hq, eps, q_out):
    """caches: (codes, scales) of keys and of values.  Returns (q_out in
    float64, [(codes, scales, exact)] of keys and values): `exact` holds the new
    positions' x / 2^(scale - 127) before rounding and saturation, NaN elsewhere;
    the codes there are its rounding."""
    P, Hkv, ps, d = caches[0][0].shape
    nothing = [np.full((P, Hkv, ps, d), np.nan) for _ in range(2)]
    q, new_k, new_v = paged_append(qkv, q_w, k_w, cos_sin, *nothing, table, start, seq_len, Hq, eps, q_out)
    blocks = {}  # (page, block) -> (slots of the new rows, whether earlier positions are there)
    for r, b, pos in rows(start, seq_len):
        at = place(table, b, pos, ps, P)
        if at is None or pos >= cos_sin.shape[0]:
            continue
        slots, before = blocks.setdefault((at[0], at[1] // BLOCK), ([], pos % BLOCK))
        slots.append(at[1])
    done = []
    for (codes, scales), new in zip(caches, (new_k, new_v)):
        codes, scales, exact = codes.copy(), scales.copy(), np.full((P, Hkv, ps, d), np.nan)
        for (page, block), (slots, before) in blocks.items():
            for g in range(Hkv):
                x = new[page, g, slots]
                s = least_scale(np.abs(x[np.isfinite(x)]).max(initial=0.0))
                if before:
                    was = clamp_scale(scales[page, g, block])
                    s = max(s, was)
                    if s > was:
                        old = codes[page, g, block * BLOCK:block * BLOCK + before]
                        again = e4m3(np.ldexp(e4m3_values()[old], was - s))
                        codes[page, g, block * BLOCK:block * BLOCK + before] = again
                if not before or clamp_scale(scales[page, g, block]) != s:
                    scales[page, g, block] = s
                exact[page, g, slots] = np.ldexp(x, 127 - s)
                codes[page, g, slots] = e4m3(exact[page, g, slots])
        done.append((codes, scales, exact))
    return q, done


# ---------------------------------------------------------------------------
# logits before sampling
# ---------------------------------------------------------------------------
def adjust_row(logits, history=(), prompt=0, repetition=1.0, frequency=0.0, presence=0.0, biases=(), mask=None):
    """float64: one row's logits after the penalties for the tokens of `history`
    (its first `prompt` the prompt's), the biases ((token, value), the last for a
    token) and the mask (words of 32 tokens)."""
    x = np.array(logits, dtype=np.float64)
    V = len(x)
    count, seen = {}, set()
    for i, t in enumerate(history):
        if 0 <= t < V:
            seen.add(int(t))
            if i >= prompt:
                count[int(t)] = count.get(int(t), 0) + 1
    with np.errstate(all="ignore"):
        for t in seen:
            x[t] = x[t] / np.float64(repetition) if x[t] > 0 else x[t] * np.float64(repetition)
        for t, c in count.items():
            x[t] = x[t] - np.float64(frequency) * c - np.float64(presence)
        for t, v in dict((int(t), v) for t, v in biases).items():
            if 0 <= t < V:
                x[t] = x[t] + np.float64(v)
    if mask is not None:
        for t in range(V):
            if not int(mask[t // 32]) >> (t % 32) & 1:
                x[t] = -np.inf
    return x
