"""The serving operators from their definitions, in numpy and 64 bits."""

import math

import numpy as np


def race(w, e):
    """Lowest index of the largest w / e; a NaN loses."""
    with np.errstate(divide="ignore", invalid="ignore"):
        r = w / e.astype(np.float64)
    return int(np.argmax(np.where(np.isnan(r), -np.inf, r)))


def draft(oracle, states, k, noise=None, temperature=1.0, last=None):
    """Tokens, states and log-probabilities; the model's scores are the oracle's fp32 ones."""
    state = np.asarray(states, np.int32).copy()
    B = len(state)
    if last is not None:
        nxt = oracle.advance(state)[1]
        state = np.where(last >= 0, nxt[np.arange(B), np.maximum(last, 0)], state).astype(np.int32)
    tokens, after, rows = [], [state], []
    for i in range(k):
        score, nxt = oracle.advance(state)[:2]
        x = score.astype(np.float64)
        if temperature:
            x = (x - x.max(1, keepdims=True)) / temperature
            w = np.exp(x)
            rows.append(x - np.log(w.sum(1, keepdims=True)))
            tok = np.array([race(w[b], noise[b, i]) for b in range(B)])
        else:
            tok = x.argmax(1)
        state = nxt[np.arange(B), tok].astype(np.int32)
        tokens.append(tok)
        after.append(state)
    return np.stack(tokens, 1), np.stack(after, 1), np.stack(rows, 1) if rows else None


def probabilities(logits, temperature):
    """softmax(logits / temperature): NaN as -inf, +inf logits share the mass, 0 where nothing is above -inf."""
    x = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    m = x.max()
    if m == -np.inf:
        return np.zeros_like(x)
    w = (x == m).astype(np.float64) if m == np.inf else np.exp((x - m) / temperature)
    return w / w.sum()


def verify(logits, tokens, logprobs=None, uniforms=None, noise=None, temperature=1.0, lengths=None):
    B, K = tokens.shape
    V = logits.shape[2]
    out, kept = np.full((B, K + 1), -1), np.zeros(B, int)
    for b in range(B):
        n = K if lengths is None else min(max(int(lengths[b]), 0), K)
        for k in range(n):
            if not 0 <= tokens[b, k] < V:
                n = k
                break
        for k in range(n + 1):
            token = int(tokens[b, k]) if k < n else -1
            if temperature == 0:
                x = np.where(np.isnan(logits[b, k]), -np.inf, logits[b, k].astype(np.float64))
                added = int(x.argmax())
                keep = k < n and added == token and x.max() > -np.inf
            else:
                p = probabilities(logits[b, k], temperature)
                q = np.zeros(V)
                if k < n:
                    q = np.exp(logprobs[b, k].astype(np.float64)) if logprobs is not None else np.eye(1, V, token)[0]
                keep = k < n and float(uniforms[b, k]) * q[token] < p[token]
                if not keep:
                    rest = np.maximum(p - q, 0)
                    rest = rest if (rest > 0).any() else p
                    added = race(rest, noise[b]) if (rest > 0).any() else 0
            if not keep:
                out[b, k], kept[b] = added, k
                break
            out[b, k] = token
    return out, kept


def rotate(x, cos, sin, layout):
    """x [..., D] turned by cos, sin [R / 2]."""
    y = x.astype(np.float64).copy()
    i = np.arange(cos.shape[-1])
    a, b = (i, i + len(i)) if layout == 0 else (2 * i, 2 * i + 1)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def attend(q, k_cache, v_cache, pages=None, lengths=None, prefix_pages=None, prefix_lengths=None, q_lengths=None,
           scale=None):
    """Output, log of the sum, and the sum of softmax times |v| (what rounding errors are relative to)."""
    S, T, Hq, D = q.shape
    P, page, H, _ = k_cache.shape
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, lse, size = np.zeros(q.shape), np.full((S, T, Hq), -np.inf), np.zeros(q.shape)

    def places(table, n):
        n = min(max(int(n), 0), len(table) * page)
        return [(int(table[j // page]), j % page) for j in range(n)]

    for s in range(S):
        prefix = [] if prefix_pages is None else places(
            prefix_pages[s // (S // len(prefix_pages))], prefix_lengths[s // (S // len(prefix_pages))])
        own = [] if pages is None else places(pages[s], lengths[s])
        nq = T if q_lengths is None else min(max(int(q_lengths[s]), 0), T)
        for t in range(nq):
            at = prefix + own[:max(0, len(own) - nq + t + 1)]
            at = [a for a in at if 0 <= a[0] < P]
            if not at:
                continue
            pg, entry = np.array(at).T
            for h in range(Hq):
                kv = h // (Hq // H)
                k, v = k_cache[pg, entry, kv], v_cache[pg, entry, kv]
                with np.errstate(invalid="ignore", over="ignore"):
                    x = k @ q[s, t, h] * scale
                    m = x.max()
                    w = np.exp(x - m)
                    lse[s, t, h] = m + np.log(w.sum())
                    out[s, t, h] = (w[:, None] * v).sum(0) / w.sum()
                    size[s, t, h] = (w[:, None] * abs(v)).sum(0) / w.sum()
    return out, lse, size
