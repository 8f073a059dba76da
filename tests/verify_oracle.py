"""The verification of drafted trees on the host, by the rule itself, request after request in 64 bits."""
import numpy as np

MOST = float(np.finfo(np.float32).max)


def weights(row):
    """A row of probabilities as they count."""
    w = np.asarray(row, dtype=np.float64)
    return np.minimum(np.where(w > 0, w, 0.0), MOST)   # NaN compares false


def verify(target, draft, tokens, parents, u, q_start, path_stride, max_nodes, lens=None, totals=None):
    """(paths, accepted, next, whether anything was out of range); rows as 64-bit arrays."""
    vocab, paths, accepted, nxt, flag = target.shape[1], [], [], [], False
    for r in range(len(q_start) - 1):
        a, b = int(q_start[r]), int(q_start[r + 1])
        n = b - a
        if n < 0 or b > len(tokens):
            flag, n = True, 0
        if lens is not None and int(totals[r]) - int(lens[r]) < n:
            n = 0
        if n > max_nodes:
            flag, n = True, max_nodes
        path, v = [], -1
        if n:
            path, ruled, c, s = [0], [], 0.0, 1.0
            p, q = weights(target[a]), None if draft is None else weights(draft[a])

            def left():
                w = p.copy() if draft is None else np.maximum(p - c * q, 0.0)
                w[ruled] = 0.0
                return w

            for i in range(1, n):
                if len(path) == path_stride or not s > 0:
                    break
                if parents[a + i] != path[-1]:
                    continue
                t = int(tokens[a + i])
                if not 0 <= t < vocab:
                    flag = True
                    continue
                w = left()[t]
                if w > 0 and float(u[a + i]) * (1.0 if draft is None else q[t]) * s < w:
                    path.append(i)
                    ruled, c, s = [], 0.0, 1.0
                    p, q = weights(target[a + i]), None if draft is None else weights(draft[a + i])
                elif draft is None:
                    ruled.append(t)
                    s = float(left().sum())
                else:
                    c += s
                    s = float(left().sum())
            w = left()
            if not w.sum() > 0:
                w = p
            if w.sum() > 0:
                run, goal = np.cumsum(w), float(u[a]) * w.sum()
                past = np.flatnonzero((run > goal) & (w > 0))
                v = int(past[0]) if len(past) else int(np.flatnonzero(w)[-1])
            else:
                flag = True
        paths.append(path + [-1] * (path_stride - len(path)))
        accepted.append(len(path))
        nxt.append(v)
    return paths, accepted, nxt, flag
