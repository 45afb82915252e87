"""Plain CPU definitions of the calls of include/rrq_draft.h, written from the
header's formulas in numpy, in 64 bits.
"""

import numpy as np

from oracle import serving

F32 = np.float32
U = 2.0 ** -24          # half a step of binary32, relative


def normed(x, kind, eps):
    """Rows of x normed, without weights."""
    if kind == "layer":
        x = x - x.mean(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        return x / np.sqrt(np.square(x).mean(1, keepdims=True) + eps)


def block_norm(residual, y, weight, bias, kind, post, post_weight, gate, scale, eps):
    """(out, h) in 64 bits."""
    h = residual.astype(np.float64)
    if y is not None:
        y = y.astype(np.float64)
        if post:
            y = normed(y, post, eps)
            if post_weight is not None:
                y = y * post_weight.astype(np.float64)
        if gate is not None:
            y = gate.astype(np.float64) * y
        h = h + scale * y
    out = normed(h, kind, eps)
    if weight is not None:
        out = out * weight.astype(np.float64)
    return (out if bias is None else out + bias.astype(np.float64)), h


def _normed_error(x, dx, kind, eps, terms):
    """How far a norm computed in binary32 may be off, for elements off by dx: sums
    round `terms` times at most, each rounding is off by U of its result."""
    if kind == "layer":
        dm = dx.mean(1, keepdims=True) + terms * U * np.abs(x).mean(1, keepdims=True)
        x = x - x.mean(1, keepdims=True)
        dx = dx + dm + U * np.abs(x)
    s = np.square(x).mean(1, keepdims=True) + eps
    # 2 |x| dx + dx^2 a term
    ds = (2 * np.abs(x) * dx + dx * dx).mean(1, keepdims=True) + terms * U * s
    with np.errstate(invalid="ignore", divide="ignore"):
        f = 1 / np.sqrt(s)
        # 1 / sqrt(s - ds) - 1 / sqrt(s) bounds both sides; the square root, the
        # quotient and the product with it round
        worst = np.where(ds < s, 1 / np.sqrt(np.maximum(s - ds, 1e-300)), np.inf)
        return dx * worst + np.abs(x) * ((worst - f) + 5 * U * f)


def block_norm_error(residual, y, weight, bias, kind, post, post_weight, gate, scale, eps):
    """(out, h): bounds of the binary32 arithmetic's errors, before results are
    rounded to their types."""
    # a thread's elements one after another (64 at most), lanes, waves; 1 / n, the
    # product with it, and eps
    terms = 64 + 6 + 16 + 3
    h = residual.astype(np.float64)
    dh = np.zeros_like(h)
    if y is not None:
        y = y.astype(np.float64)
        dy = np.zeros_like(y)
        if post:
            dy = _normed_error(y, dy, post, eps, terms)
            y = normed(y, post, eps)
            if post_weight is not None:
                w = post_weight.astype(np.float64)
                y, dy = y * w, dy * np.abs(w)
                dy = dy + U * np.abs(y)
        if gate is not None:
            g = gate.astype(np.float64)
            y, dy = y * g, dy * np.abs(g)
            dy = dy + U * np.abs(y)
        y, dy = scale * y, abs(scale) * dy
        dy = dy + U * np.abs(y)
        h = h + y
        dh = dy + U * np.abs(h)
    d = _normed_error(h, dh, kind, eps, terms)
    out = normed(h, kind, eps)
    if weight is not None:
        w = weight.astype(np.float64)
        out, d = out * w, d * np.abs(w)
        d = d + U * np.abs(out)
    if bias is not None:
        out = out + bias
        d = d + U * np.abs(out)
    # (products of two errors, and what binary32 loses below its range)
    return d * 1.01 + 1e-37, dh * 1.01 + 1e-37


def rotate(x, positions, frequencies, layout, amplitude):
    """Rows x [tokens, heads, dim] (binary32) rotated, each operation rounded to
    binary32; cosines and sines are rounded once."""
    rot = 2 * len(frequencies)
    angle = np.asarray(positions, np.float64)[:, None] * frequencies
    c, s = ((amplitude * f(angle)).astype(F32)[:, None] for f in (np.cos, np.sin))
    x = np.asarray(x, F32)
    pick = ((slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else
            (slice(0, rot, 2), slice(1, rot, 2)))
    a, b = x[..., pick[0]], x[..., pick[1]]
    out = x.copy()
    out[..., pick[0]] = a * c - b * s
    out[..., pick[1]] = b * c + a * s
    return out


def places(lengths, offsets):
    """Each row's place in its sequence."""
    return [length - (offsets[b + 1] - offsets[b]) + i for b, length in enumerate(lengths)
            for i in range(offsets[b + 1] - offsets[b])]


def append(cache, table, lengths, offsets, positions, frequencies, layout, amplitude, Q, K, V):
    """The rotated queries (binary32); keys and values are written in place."""
    if positions is None:
        positions = places(lengths, offsets)
    turn = (positions, frequencies, layout, amplitude)
    serving.write(cache, table, lengths, offsets, rotate(K, *turn), V)
    return rotate(Q, *turn)


def tree_attention(cache, table, lengths, offsets, Q, seen, positions, scale, window=0):
    """(out, weight, reach) as serving.attention; seen: for each row the set of its
    step's rows that it sees."""
    T, Hq, D = Q.shape
    ratio = Hq // cache.k.shape[1]
    out, mean_abs = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    reach = np.zeros((T, Hq))
    for b, length in enumerate(lengths):
        n = offsets[b + 1] - offsets[b]
        start = length - n
        for h in range(Hq if n > 0 else 0):
            k = serving.dense(cache, table[b], "k", h // ratio, length)
            v = serving.dense(cache, table[b], "v", h // ratio, length)
            for i in range(n):
                row = offsets[b] + i
                p = start + i if positions is None else positions[row]
                keys = [j for j in range(max(start, 0)) if not window or j > p - window]
                keys += [start + j for j in sorted(seen[row]) if j < n and start + j >= 0]
                if not keys:
                    continue
                q = Q[row, h].astype(np.float64)
                s = scale * (k[keys] @ q)
                w = np.exp(s - s.max())
                w /= w.sum()
                out[row, h] = w @ v[keys]
                mean_abs[row, h] = w @ np.abs(v[keys])
                reach[row, h] = (np.abs(k[keys]) @ np.abs(q)).max()
    return out, mean_abs, reach


def _softmax(x, temperature):
    """Probabilities of logits x in 64 bits; at a temperature of 0 the first largest."""
    x = np.asarray(x, np.float64)
    if temperature == 0:
        p = np.zeros_like(x)
        if not np.isnan(x).all():       # (np.nanargmax takes a NaN for -inf)
            p[int(np.nonzero(x == np.nanmax(x))[0][0])] = 1.0
        return p
    if np.isnan(x).any() or not np.isfinite(x.max()):
        return np.full_like(x, np.nan)
    p = np.exp((x - x.max()) / temperature)
    return p / p.sum()


def verify(logits, tokens, offsets, max_accept, uniforms, draft=None, parents=None,
           temperature=1.0, draft_temperature=1.0):
    """(counts, following, paths, margin): margin is how near, relative, any acceptance
    came to its border; for the token drawn, 10^6 times the share of the whole between
    the random number and the nearer border (its sums are that much finer)."""
    counts, following, paths = [], [], []
    margin = np.inf
    vocab = logits.shape[1]
    for b in range(len(offsets) - 1):
        o, n = offsets[b], max(0, offsets[b + 1] - offsets[b])
        path = [0] if n else []
        p = _softmax(logits[o], temperature) if n else None
        j = 1
        while j < n and len(path) <= max_accept:
            i = path[-1]
            parent = j - 1 if parents is None else int(parents[o + j])
            if parent != i:
                j += 1
                continue
            t, u = int(tokens[o + j]), float(uniforms[o + j])
            inside = 0 <= t < vocab
            if draft is not None and temperature > 0:
                q = _softmax(draft[b, j - 1], draft_temperature)
                left, right = u * (q[t] if inside else 0.0), p[t] if inside else 0.0
                if left < right:
                    margin = min(margin, (right - left) / max(right, 1e-300))
                    path.append(j)
                    p = _softmax(logits[o + j], temperature)
                    j += 1
                    continue
                margin = min(margin, (left - right) / left if left > 0 else np.inf)
                rest = np.clip(p - q, 0, None)
                p = rest if np.nansum(rest) > 0 else p
                break
            left, right = u * p.sum(), p[t] if inside else 0.0
            if left < right:
                margin = min(margin, (right - left) / right)
                path.append(j)
                p = _softmax(logits[o + j], temperature)
            else:
                if temperature > 0 and left > 0:
                    margin = min(margin, (left - right) / left)
                if inside and temperature > 0:
                    p = p.copy()
                    p[t] = 0.0
            j += 1
        counts.append(max(len(path) - 1, 0))
        nxt = -1
        if n and temperature == 0:
            nxt = int(np.argmax(p)) if p.sum() > 0 else -1
        elif n and np.isfinite(p.sum()) and p.sum() > 0:
            total = np.cumsum(p)
            goal = float(uniforms[o]) * total[-1]
            above = np.nonzero(total > goal)[0]
            nxt = int(above[0]) if len(above) else int(np.nonzero(p)[0][-1])
            margin = min(margin, (total[nxt] - goal) / total[-1] * 1e6,
                         (goal - (total[nxt] - p[nxt])) / total[-1] * 1e6
                         if total[nxt] > p[nxt] else np.inf)
        following.append(nxt)
        paths.append(path + [-1] * (max_accept + 1 - len(path)))
    return np.array(counts), np.array(following), np.array(paths), margin
