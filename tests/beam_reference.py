"""The beam search's operators from their definitions, one after the other, in plain Python and numpy."""

import numpy as np


def fork(pages, lengths, parents, refs, page, tokens):
    """Rows, lengths, copies and counts after a fork; ``pages`` [G * W, width], ``parents`` and ``tokens`` [G, K]."""
    (G, K), width, P = parents.shape, pages.shape[1], len(refs)
    W, refs = len(pages) // G if G else 0, [int(r) for r in refs]

    def count(row, by):
        for p in row:
            if 0 <= p < P:
                refs[p] += by
    rows, sizes, wants = [], [], []
    for g in range(G):
        for j in range(K):
            w = int(parents[g, j])
            live = 0 <= w < W
            n = min(max(int(lengths[g * W + w]), 0), width * page) if live else None
            rows.append([int(p) for p in pages[g * W + w, :-(-n // page)]] if live else [])
            sizes.append(n)
            wants.append(max(int(tokens[g, j]), 0))
    for row in pages.tolist():
        count(row, -1)
    for row in rows:
        count(row, 1)
    free = [p for p in range(P) if refs[p] == 0]
    after_step1 = list(refs)
    decided, plans = {}, []
    for i, (row, n, T) in enumerate(zip(rows, sizes, wants)):
        if n is None or n + T > width * page:
            plans.append((False, 0))
            continue
        shared = False
        if T > 0 and n % page and 0 <= row[-1] < P:
            key = i // K, row[-1]
            shared = after_step1[row[-1]] - decided.get(key, 0) > 1
            decided[key] = decided.get(key, 0) + 1
        plans.append((shared, -(-(n + T) // page) - len(row) if T > 0 else 0))
    taken, out, after, copies = 0, [], [], []
    for row, n, T, (shared, more) in zip(rows, sizes, wants, plans):
        need = int(shared) + more
        mine = free[taken:taken + need]
        taken += need
        if n is not None and (n + T > width * page or need > 0 and taken > len(free)):
            count(row, -1)
            row, n, shared, mine = [], -1, False, []
        copies.append((row[-1], mine[0], n % page) if shared else (-1, -1, 0))
        if shared:
            count(row[-1:], -1)
            row = row[:-1]
        count(mine, 1)
        row = row + mine
        out.append(row + [-1] * (width - len(row)))
        after.append(n or 0)
    i32 = np.int32
    return (np.array(out, i32).reshape(G * K, width), np.array(after, i32), np.array(copies, i32).reshape(G * K, 3),
            np.array(refs, i32))


def compact(refs, page, tables):
    """Copies, new numbers, counts and tables after a compaction."""
    refs = [int(r) for r in refs]
    P = len(refs)
    used = [p for p in range(P) if refs[p]]
    holes = [p for p in range(len(used)) if not refs[p]]
    moved, copies = list(range(P)), []
    for p in used[len(used) - len(holes):]:
        moved[p] = holes[len(copies)]
        copies.append((p, moved[p], page))
    for p, to, _ in copies:
        refs[to], refs[p] = refs[p], 0
    copies += [(-1, -1, 0)] * (P // 2 - len(copies))
    new = [np.array([moved[p] if 0 <= p < P else p for p in t.flatten().tolist()], np.int32).reshape(t.shape)
           for t in tables]
    return np.array(copies, np.int32).reshape(P // 2, 3), np.array(moved, np.int32), np.array(refs, np.int32), new


def copy(cache, copies):
    """A cache [pages, page size, ...] after the copies."""
    out = cache.copy()
    for src, dst, entries in np.asarray(copies).tolist():
        if 0 <= src < len(cache) and 0 <= dst < len(cache) and src != dst:
            n = min(max(entries, 0), cache.shape[1])
            out[dst, :n] = cache[src, :n]
    return out


def e4m3_values():
    """The value of each byte: sign, 4 bits of exponent (bias 7), 3 of mantissa, 0x7f and 0xff no number."""
    b = np.arange(256)
    e, m = b >> 3 & 15, b & 7
    x = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e.astype(float) - 7))
    x[b & 0x7f == 0x7f] = np.nan
    return np.where(b & 0x80, -x, x)


_LEVELS = e4m3_values()[:127]


def to_e4m3(x):
    """The nearest e4m3 value of each |x| <= 464, of two the one with an even mantissa; no number for what is not finite."""
    with np.errstate(invalid="ignore"):
        a = np.abs(x)
        hi = np.clip(np.searchsorted(_LEVELS, a), 1, 126)
        lo = hi - 1
        below, above = a - _LEVELS[lo], _LEVELS[hi] - a
        pick = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
        return np.where(np.isfinite(x), np.copysign(_LEVELS[pick], x), np.nan)


def append8(x, cache, scale, pages, start, counts):
    """``cache`` [pages, page, heads, dim] of e4m3 values and ``scale`` [pages, blocks, heads] after x [S, T, heads, dim]
    in fp32; and which entries are new or kept."""
    cache, scale = cache.copy(), scale.copy()
    P, page, H, D = cache.shape
    block = page // scale.shape[1]
    known = np.zeros(cache.shape[:2], bool)
    for s in range(len(x)):
        groups = {}
        for t in range(counts[s]):
            place = int(start[s]) + t
            if 0 <= place < pages.shape[1] * page and 0 <= pages[s, place // page] < P:
                groups.setdefault((place // block, int(pages[s, place // page])), []).append((place, t))
        for (b, p), new in groups.items():
            at = b * block % page // block
            lead = new[0][0] % block
            first = b * block % page
            for h in range(H):
                y = x[s, [t for _, t in new], h].astype(np.float32)
                most = np.where(np.isfinite(y), np.abs(y), 0).max()
                e = -100
                while np.float64(most) > 448 * 2.0 ** e:
                    e += 1
                now = np.float32(2.0 ** e)
                if lead:
                    old = scale[p, at, h]
                    old = old if 2.0 ** -100 <= old < np.inf else np.float32(2.0 ** -100)
                    if most > np.float32(448) * old:
                        ratio = np.float32(old) / now
                        cache[p, first:first + lead, h] = to_e4m3(cache[p, first:first + lead, h].astype(np.float32) * ratio)
                    else:
                        now = old
                scale[p, at, h] = now
                with np.errstate(invalid="ignore"):
                    cache[p, first + lead:first + lead + len(new), h] = to_e4m3(y * (np.float32(1) / now))
            known[p, first:first + lead + len(new)] = True
    return cache, scale, known


def beam_step(oracle, V, asr, lam, states, scores, k, mode="plain", last=None):
    """Classes, parents, sums and states of the k best continuations.  The sums are the operator's own fp32 ones: one
    rounding of asr + lam * lm (through 64 bits of mantissa, which the 48 of the product fit) and one of the sum."""
    B, W = states.shape
    C = V + (mode != "plain")
    out = np.full((B, k), -1, np.int32), np.full((B, k), -1, np.int32), np.full((B, k), -np.inf, np.float32), \
        np.zeros((B, k), np.int32)
    bad = 0
    for b in range(B):
        total, after = np.full((W, C), -np.inf, np.float32), np.zeros((W, C), np.int32)
        for w in range(W):
            if not scores[b, w] > -np.inf:
                continue
            s = int(states[b, w])
            if last is not None and last[b, w] == V:
                total[w, V], after[w, V] = scores[b, w], s
                continue
            if not 0 <= s < oracle.num_states:
                bad += 1
                continue
            lm, to = oracle.advance(np.array([s], np.int32))[:2]
            lm, to = lm[0], to[0]
            if mode != "plain":
                end = oracle.final(np.array([s], np.int32))[0] if mode == "aed" else np.float32(0)
                lm, to = np.append(lm, np.float32(end)), np.append(to, s)
            with np.errstate(invalid="ignore", over="ignore"):
                fused = (np.longdouble(np.float32(lam)) * lm.astype(np.longdouble) + asr[b, w, :C]).astype(np.float32)
                total[w] = scores[b, w] + fused
            after[w] = to
        flat = np.where(np.isnan(total), -np.inf, total).ravel()
        for j, i in enumerate(np.argsort(-flat, kind="stable")[:k]):
            if flat[i] > -np.inf:
                out[1][b, j], out[0][b, j] = divmod(int(i), C)
                out[2][b, j], out[3][b, j] = flat[i], after.ravel()[i]
    return (*out, bad)
