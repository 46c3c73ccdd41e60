"""Plain statement of kvb_accept for the tests: one request, one draft, one token at a time, every operation rounded to fp32 by itself
and sums as Python integers."""
import numpy as np

f32 = np.float32


def weights(r):
    w = np.where(r > 0, np.minimum(r, f32(1)), f32(0)).astype(f32)
    return np.floor(w * f32(2.0 ** 48)).astype(np.int64)   # (powers of two: exact)


def accept(n, parent, tokens, target, draft, u, s):
    """One request: n drafts, parent [T] or None, tokens [T], target [T+1, V], draft [T, V] or None (all fp32), u [T], s.
    Returns (path [T], accepted, token)."""
    T, V = len(tokens), target.shape[1]
    place, mass, path, r = -1, f32(1), [], target[0].copy()
    for i in range(n):
        up = i - 1 if parent is None else int(parent[i])
        up = up if -1 <= up < i else -1
        if up != place:
            continue
        x, known = int(tokens[i]), 0 <= int(tokens[i]) < V
        q = f32(1) if draft is None else draft[i, x] if known else f32(0)
        if known and f32(f32(u[i] * q) * mass) < r[x]:
            path.append(i)
            place, mass, r = i, f32(1), target[i + 1].copy()
        elif draft is None:
            if known:
                left = f32(mass - r[x])
                mass = f32(0) if left < 0 else left
                r[x] = 0
        else:
            left = (r - (mass * draft[i]).astype(f32)).astype(f32)
            r = np.where(left < 0, f32(0), left).astype(f32)
            mass = f32(float(int(weights(r).sum())) * 2.0 ** -48)
    w = weights(r)
    if int(w.sum()) == 0:
        w = weights(target[place + 1])
    total = int(w.sum())
    token = -1
    if total:
        aim = int(np.floor(np.float64(f32(s)) * np.float64(total)))
        token = int(np.searchsorted(np.cumsum(w), aim, side="right"))
    return np.array(path + [-1] * (T - len(path)), np.int32), len(path), token
