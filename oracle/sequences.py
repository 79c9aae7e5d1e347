"""float64 values of the operators over packed token rows, written from their definitions in numpy, one row
and one head at a time; and the error that fp32 arithmetic and given roundings may add to them.

A batch: q_start [seqs + 1], kv_len [seqs], table [seqs, max_pages] (ints); caches [pages, kv_heads, page, d].
Values that must not be read are marked by NaN in the tests' buffers, so nothing here reads them either."""
from __future__ import annotations

import math

import numpy as np

E32 = 2.0 ** -24                                     # half a step of fp32
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def place(table, seq, pos, page, pages):
    """(page, slot) of the token at `pos`, None if it has none."""
    if pos < 0 or pos // page >= table.shape[1]:
        return None
    p = int(table[seq, pos // page])
    return (p, pos % page) if 0 <= p < pages else None


def tokens_of(q_start, kv_len, tokens, capacity):
    """(row, sequence, position, first position of the sequence, its keys) of every row that belongs to one."""
    for s in range(len(kv_len)):
        q0 = min(max(int(q_start[s]), 0), tokens)
        q1 = min(max(int(q_start[s + 1]), q0), tokens)
        n = min(max(int(kv_len[s]), 0), capacity)
        for r in range(q0, q1):
            yield r, s, n - (q1 - q0) + (r - q0), n - (q1 - q0), n


# ------------------------------------------------------------------ block norm
def block_norm(x, residual=None, post=None, post_bias=None, gate=None, gate_act="none", scale=1.0, pre=None,
               pre_bias=None, norm="rms", eps=1e-5, half_step=0.0):
    """(y, z, bound of y, bound of z): bounds of what fp32 sums (n / 64 values of a lane in order, then a few
    of its peers), a few fp32 operations per value and the outputs' rounding can be off by."""
    n = x.shape[1]
    d = (n / 64 + 24) * E32

    def normed(v, err, w, b):
        mean = v.mean(1, keepdims=True) if norm == "layer" else 0.0
        # the mean is off by its terms' errors and its sum's
        emean = err.mean(1, keepdims=True) + d * np.abs(v).mean(1, keepdims=True) if norm == "layer" else 0.0
        c = v - mean
        ec = err + emean + E32 * np.abs(c)
        var = (c * c).mean(1, keepdims=True)
        rstd = 1.0 / np.sqrt(var + eps)
        # sum of squares: 2 |c| ec + ec^2 per term, and its sum's error; 1 / sqrt halves it, to first order
        # and, while the error is below half of the sum, by twice that
        evar = (2 * np.abs(c) * ec + ec * ec).mean(1, keepdims=True) + d * var
        erel = np.minimum(evar / (var + eps), 1.0) + 4 * E32
        out = c * rstd * w
        e = (ec * rstd + np.abs(c) * rstd * erel) * np.abs(w) + 4 * E32 * np.abs(out)
        if b is not None:
            out = out + b
            e = e + E32 * np.abs(out)
        return out, e

    u, e = x.copy(), np.zeros_like(x)
    if post is not None:
        u, e = normed(u, e, post, post_bias)
    if gate is not None:
        g = gate
        if gate_act in ("silu", "sigmoid"):
            with np.errstate(over="ignore"):
                s = 1.0 / (1.0 + np.exp(-gate))
            # exp's own error (2 units), its argument exact; 1 + e, 1 / .: half a unit each
            g = s if gate_act == "sigmoid" else gate * s
        u, e = u * g, e * np.abs(g) + 8 * E32 * np.abs(u * g)
    y = scale * u
    e = np.abs(scale) * e + 2 * E32 * np.abs(y)
    if residual is not None:
        y = residual + y
        e = e + E32 * np.abs(y)
    z = ez = None
    if pre is not None:
        z, ez = normed(y, e, pre, pre_bias)
        ez = ez * (1 + half_step) + half_step * np.abs(z) + 2.0 ** -25  # (fp16 subnormals: half a step of 2^-24)
    return y, z, e * (1 + half_step) + half_step * np.abs(y) + 2.0 ** -25, ez


# ---------------------------------------------------------------------- rotary
def rotate(head, pos, freq, interleaved, scale):
    """One head turned; and what fp32 may add: sine and cosine within 2^-22, three operations."""
    rot = 2 * len(freq)
    out, err = head.copy(), np.zeros_like(head)
    a = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    c, s = np.cos(pos * freq) * scale, np.sin(pos * freq) * scale
    u, v = head[a[0]], head[a[1]]
    out[a[0]], out[a[1]] = u * c - v * s, v * c + u * s
    err[a[0]] = err[a[1]] = (2.0 ** -22 + 4 * E32) * abs(scale) * (np.abs(u) + np.abs(v))
    return out, err


def rotary(x, freq, q_start, kv_len, heads, kv_heads, d, table=None, page=1, pages=0, interleaved=False, scale=1.0):
    """Dicts {row: (queries, bound)} and {(page, slot): (keys, bound, values)}."""
    q, kv = {}, {}
    cap = page * table.shape[1] if table is not None else 1 << 30
    for r, s, pos, _, _ in tokens_of(q_start, kv_len, x.shape[0], cap):
        row = x[r].reshape(heads + 2 * kv_heads, d)
        turned = [rotate(row[h], pos, freq, interleaved, scale) for h in range(heads + kv_heads)]
        q[r] = (np.concatenate([t[0] for t in turned[:heads]]), np.concatenate([t[1] for t in turned[:heads]]))
        at = place(table, s, pos, page, pages) if kv_heads else None
        if at is not None:
            kv[at] = (np.stack([t[0] for t in turned[heads:]]), np.stack([t[1] for t in turned[heads:]]), row[heads + kv_heads:])
    return q, kv


# ------------------------------------------------------------------- attention
def attention(x, k, v, q_start, kv_len, table, heads, scale=None, causal=True, window=0, max_q=None, half_step=0.0,
              p_step=0.0, stride=1):
    """{row: (output, bound)} of the rows that belong to a sequence (every stride-th).  p_step: what the
    probabilities are rounded by before the second product.

    Bound, with A = sum p |v| / sum p: a score is off by (d + 3) E32 sum |q k| scale (d sums in any order, its
    scaling, the subtraction of the maximum) and E32 times the exponent's size, the power itself by 2 units; the
    sums run over N terms in any order, and the running factors round N / 32 times at most."""
    pages, kv_heads, page, d = k.shape
    g = heads // kv_heads
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = {}
    seen_of = {}
    for n_row, (r, s, pos, pos0, n) in enumerate(tokens_of(q_start, kv_len, x.shape[0], page * table.shape[1])):
        if max_q is not None and pos - pos0 >= max_q:
            continue
        if n_row % stride:
            continue
        lo = max(0, pos - window + 1) if window else 0
        hi = min(n, pos + 1) if causal else n
        keys = []
        for j in range(lo, hi, 1):
            at = place(table, s, j, page, pages)
            if at is not None:
                keys.append(at)
        o = np.zeros((heads, d))
        e = np.zeros((heads, d))
        if keys:
            pi, si = np.array([a[0] for a in keys]), np.array([a[1] for a in keys])
            row = x[r].reshape(heads, d)
            for h in range(heads):
                kk, vv = k[pi, h // g, si], v[pi, h // g, si]
                with np.errstate(invalid="ignore", over="ignore"):
                    sc = scale * (kk @ row[h])
                    w = np.exp(sc - sc.max())
                    o[h] = (w @ vv) / w.sum()
                    size = scale * (np.abs(kk) @ np.abs(row[h])).max()
                    span = float(sc.max() - sc.min())
                    rel = 2 * ((d + 3) * E32 * size + E32 * span + 4 * E32) + 2 * (len(keys) + len(keys) / 32 + 8) * E32 + p_step
                    e[h] = rel * (w @ np.abs(vv)) / w.sum()
        out[r] = (o.reshape(-1), e.reshape(-1) * (1 + half_step) + half_step * np.abs(o).reshape(-1) + 2.0 ** -25)
    return out
