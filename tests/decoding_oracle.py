"""The decoding step's choices from their definitions, in 64 bits on the host (numpy): what include/nms.h says, entry by entry.
Written for being read; the GPU results have to equal it."""
import numpy as np


def probabilities(row):
    row = np.asarray(row, np.float64)
    return np.where(np.isfinite(row) & (row > 0), row, 0.0)


def verify(target, draft, drafts, counts, uniforms):
    """target [S][K+1][V], draft [S][K][V] or None, drafts [S][K], counts [S] or None, uniforms [S][K+1] (float32 values).
    Returns tokens [S][K+1] and accepted [S]."""
    s, k1, v = target.shape
    tokens, accepted = np.full((s, k1), -1, np.int32), np.zeros(s, np.int32)
    for i in range(s):
        count = k1 - 1 if counts is None else min(int(counts[i]), k1 - 1)
        if count < 0:
            continue
        a = 0
        while a < count:
            x = int(drafts[i, a])
            inside = 0 <= x < v
            p = probabilities(target[i, a, x]) if inside else 0.0
            q = 1.0 if draft is None else (probabilities(draft[i, a, x]) if inside else 0.0)
            if not (np.float64(uniforms[i, a]) * q < p):
                break
            tokens[i, a] = x
            a += 1
        p = probabilities(target[i, a])
        w = p
        if a < count:
            if draft is None:
                w = p.copy()
                x = int(drafts[i, a])
                if 0 <= x < v:
                    w[x] = 0.0
            else:
                w = np.maximum(p - probabilities(draft[i, a]), 0.0)
            if not w.any():
                w = p
        accepted[i] = a
        if not w.any():
            continue
        c = np.cumsum(w)
        past = np.flatnonzero((c > np.float64(uniforms[i, -1]) * c[-1]) & (w > 0))
        tokens[i, a] = past[0] if past.size else np.flatnonzero(w)[-1]
    return tokens, accepted


def add_weights(sums, weights, counts, valid):
    """sums [S][H][N] float32 plus weights [S][H][G][T][C] (float64 values), rounded once."""
    out = sums.copy()
    if weights is None:
        return out
    s, h, g, t, c = weights.shape
    n_max = sums.shape[-1]
    for i in range(s):
        n = min(n_max if counts is None else int(np.clip(counts[i], 0, n_max)), c)
        total = sums[i, :, :n].astype(np.float64)
        for a in range(g):
            for b in range(t if valid is None else int(np.clip(valid[i], 0, t))):
                w = weights[i, :, a, b, :n]
                total = total + np.where(np.isfinite(w), w, 0.0)
        out[i, :, :n] = total.astype(np.float32)
    return out


def keep(sums, positions, counts, lengths, budget, first, recent):
    """The keep vector [S][H][N], kept [S] and the moves [S][H] -> list of (to, from)."""
    s, h, n_max = sums.shape
    out, kept, moves = np.zeros((s, h, n_max), np.uint8), np.zeros(s, np.int32), []
    for i in range(s):
        n = n_max if counts is None else int(np.clip(counts[i], 0, n_max))
        length = n if lengths is None else int(lengths[i])
        k = kept[i] = min(n, budget)
        for j in range(h):
            p = np.arange(n) if positions is None else positions[i, j, :n].astype(np.int64)
            guarded = (p < first) | (p >= length - recent)
            with np.errstate(invalid="ignore"):
                held = sums[i, j, :n].astype(np.float64)
            lost = np.isnan(held)
            held = np.where(lost | guarded, 0.0, held)
            order = np.lexsort((np.arange(n), -held, lost & ~guarded, ~guarded))
            out[i, j, order[:k]] = 1
            free, moved = np.flatnonzero(out[i, j, :k] == 0), k + np.flatnonzero(out[i, j, k:n])
            moves.append(list(zip(free.tolist(), moved.tolist())))
    return out, kept, [moves[i * h:(i + 1) * h] for i in range(s)]


def evict(sums, positions, counts, lengths, weights, valid, budget, first, recent, tensors):
    """The whole path on tensors [S][H][N][...]; returns new (keep, kept, sums, positions, tensors)."""
    sums = add_weights(sums, weights, counts, valid)
    flags, kept, moves = keep(sums, positions, counts, lengths, budget, first, recent)
    new_sums, new_positions = sums.copy(), None if positions is None else positions.copy()
    new_tensors = [t.copy() for t in tensors]
    for i in range(sums.shape[0]):
        n = sums.shape[2] if counts is None else int(np.clip(counts[i], 0, sums.shape[2]))
        for j in range(sums.shape[1]):
            for to, fro in moves[i][j]:
                new_sums[i, j, to] = sums[i, j, fro]
                if positions is not None:
                    new_positions[i, j, to] = positions[i, j, fro]
                for t, old in zip(new_tensors, tensors):
                    t[i, j, to] = old[i, j, fro]
            new_sums[i, j, kept[i]:n] = 0.0
    return flags, kept, new_sums, new_positions, new_tensors
