"""fp64 references of the speculative step: norm and rotation of Q and K, attention of drafted trees, verification
(test infrastructure only; plain loops over rows, numpy)."""
import math

import numpy as np


def ref_rope(x, positions, inv_freq, rotary_dim, interleaved=False, norm=None, eps=0.0, axis_pairs=None):
    """x [T, H, D], positions [axes][T] -> (float64 [T, H, D], the sizes |a| + |b| of the pair behind each feature).

    y = x * norm / sqrt(mean x^2 + eps); pair i of y turns by positions[axis of i] * inv_freq[i]."""
    x = np.asarray(x, np.float64)
    y = x if norm is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(norm, np.float64)
    out, size = y.copy(), np.abs(y)
    pairs = rotary_dim // 2
    axis = np.zeros(pairs, int) if axis_pairs is None else np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        angle = [math.remainder(float(p) * float(inv_freq[i]), 2 * math.pi) for p in positions[axis[i]]]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size


def ancestors(parents):
    """bool [n, n]: whether node j is i or an ancestor of it."""
    seen = np.eye(len(parents), dtype=bool)
    for i, p in enumerate(parents):
        if p >= 0:
            seen[i] |= seen[p]
    return seen


def mask_words(seen, words):
    """int64 [n, words] of bool [n, m]."""
    out = np.zeros((seen.shape[0], words), np.uint64)
    for i, j in zip(*np.nonzero(seen)):
        out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out.view(np.int64)


def ref_tree_attention(q, k, v, seen, scale, step, half):
    """One sequence: q [n, Hq, D], k, v [ctx + n, Hkv, D], seen bool [n, n] -> (float64 [n, Hq, D], how far a result in 16 bits may be off).

    step: half a step of the element type, relative (2^-8, 2^-11); half: whether it is fp16, whose weights below 2^-14 are
    rounded to multiples of 2^-24.  The bound, for weights w (sum 1) of which each is rounded once and is off by
    its score's error e besides: |sum w (V - out)| * (step + e) <= (step + e) (sum w |V| + |out|), and the rounding of out."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, Hq, D = q.shape
    keys, Hkv, _ = k.shape
    ctx = keys - n
    sees = np.concatenate([np.ones((n, ctx), bool), seen], 1)
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(n):
        at = np.nonzero(sees[i])[0]
        if len(at) == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            with np.errstate(invalid="ignore", over="ignore"):
                x = scale * (k[at, g] @ q[i, h])
                off = scale * np.max(np.abs(k[at, g]) @ np.abs(q[i, h])) * D * 2.0 ** -24 + 2.0 ** -20
                w = np.exp(x - x.max())
                total = w.sum()
                y = (w / total) @ v[at, g]
                size = (w / total) @ np.abs(v[at, g]) + np.abs(y)
                t = (step + off) * size + step * np.abs(y)
                if half:
                    t = t + 2.0 ** -25 * (np.abs(v[at, g]).sum(0) + len(at) * np.abs(y)) / total + 2.0 ** -25
            out[i, h], tol[i, h] = y, t
    return out, tol


def ref_verify(tokens, parents, p, q, u, u_next):
    """One sequence of n nodes: tokens, u [n], parents [n], p, q [n, V] (q None: fixed guesses) -> (path, tokens of the step)."""
    n, vocab = len(tokens), p.shape[1]
    at, path = 0, [0]
    clean = lambda x: np.where(np.isnan(x), 0.0, np.maximum(x, 0.0))  # noqa: E731
    while True:
        row = clean(np.asarray(p[at], np.float64))
        draft = None if q is None else clean(np.asarray(q[at], np.float64))
        left, z, c, went = row.copy(), 1.0, 0.0, None
        for j in range(at + 1, n):
            if parents[j] != at:
                continue
            x = int(tokens[j])
            inside = 0 <= x < vocab
            r = left[x] if inside else 0.0
            bar = float(u[j]) * z if draft is None else float(u[j]) * (draft[x] if inside else 0.0) * z
            if bar < r and r > 0:
                went = j
                break
            if draft is None:
                z -= r
                if inside:
                    left[x] = 0.0
            else:
                c += z
                left = clean(row - c * draft)
                z = left.sum()
        if went is None:
            break
        at = went
        path.append(at)
    if not (left > 0).any():
        left = row
    run = np.cumsum(left)
    hit = np.nonzero((run > float(u_next) * run[-1]) & (left > 0))[0]
    some = np.nonzero(left > 0)[0]
    last = int(hit[0]) if len(hit) else int(some[-1]) if len(some) else -1
    return path, [int(tokens[j]) for j in path[1:]] + [last]
