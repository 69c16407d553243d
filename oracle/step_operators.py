"""Oracle for the training operators around the FFN half of the block, CPU test
infrastructure only: causal attention of ragged rows with a window and sinks, the
gated residual with the norm that follows, the global gradient norm, and their
gradients.  Plain numpy in float64, one row at a time where that is plainest.
Shares no code with the HIP path."""
import numpy as np


def visible(nq, n, window, sinks):
    """[nq, n]: whether query j, at position n - nq + j, sees the key at position x."""
    p, x = n - nq + np.arange(nq)[:, None], np.arange(n)[None, :]
    return (x <= p) & (True if window is None else (p - x < window) | (x < sinks))


def attention(q, k, v, window=None, sinks=0, scale=None, do=None):
    """One sequence: q [nq, heads, width], k and v [n, kv_heads, width]; the last query stands at the last key.
    Returns a dict of o, the weights p ([heads, nq, n]) and, given do, the gradients.  What is not visible takes no
    part, whatever its values."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    (nq, heads, width), (n, kv) = q.shape, k.shape[:2]
    scale = width ** -0.5 if scale is None else scale
    seen = visible(nq, n, window, sinks)
    some = seen.any(1)
    out = {"o": np.zeros(q.shape), "p": np.zeros((heads, nq, n))}
    if do is not None:
        do = np.asarray(do, np.float64)
        out.update(dq=np.zeros(q.shape), dk=np.zeros(k.shape), dv=np.zeros(v.shape))
    for h in range(heads):
        c = h // (heads // kv)
        with np.errstate(invalid="ignore"):
            s = np.where(seen, scale * (q[:, h] @ k[:, c].T), -np.inf)
            w = np.where(seen, np.exp(s - np.where(some, s.max(1, initial=-np.inf), 0.0)[:, None]), 0.0)
            w = w / np.where(some, w.sum(1), 1.0)[:, None]
        out["p"][h] = w
        out["o"][:, h] = unseen_apart(w, seen, v[:, c])
        if do is None:
            continue
        with np.errstate(invalid="ignore"):
            dp = do[:, h] @ v[:, c].T
            ds = np.where(seen, w * (dp - (do[:, h] * out["o"][:, h]).sum(1, keepdims=True)), 0.0)
        out["dq"][:, h] = scale * unseen_apart(ds, seen, k[:, c])
        out["dk"][:, c] += scale * unseen_apart(ds.T, seen.T, q[:, h])
        out["dv"][:, c] += unseen_apart(w.T, seen.T, do[:, h])
    return out


def unseen_apart(w, seen, rows):
    """w @ rows over the pairs that see each other alone: elsewhere 0 times infinity is 0."""
    with np.errstate(invalid="ignore"):
        if np.isfinite(rows).all() and np.isfinite(w).all():
            return w @ rows
        return np.stack([(w[i][seen[i]][:, None] * rows[seen[i]]).sum(0) for i in range(len(w))])


def scale_of_rows(table, group, rows, d):
    """1 + table[group] of each row; 1 where the row's group is none of the table's."""
    out = np.ones((rows, d))
    if table is not None:
        table = np.asarray(table, np.float64).reshape(-1, d)
        for r in range(rows):
            g = 0 if group is None else int(group[r])
            if 0 <= g < len(table):
                out[r] += table[g]
    return out


def residual_norm(x, y, alpha, gamma, group, eps, post, dh=None, dz=None):
    """h = x + (1 + alpha[group]) t, t = y, or y over its root mean square; z = h over its own, times 1 + gamma[group]."""
    x, y = np.asarray(x, np.float64), np.asarray(y, np.float64)
    rows, d = x.shape
    a, c = scale_of_rows(alpha, group, rows, d), scale_of_rows(gamma, group, rows, d)
    ry = 1 / np.sqrt((y ** 2).mean(1, keepdims=True) + eps) if post else np.ones((rows, 1))
    t = y * ry
    h = x + a * t
    r = 1 / np.sqrt((h ** 2).mean(1, keepdims=True) + eps)
    out = {"h": h, "z": h * r * c, "t": t, "r": r, "ry": ry, "a": a, "c": c}
    if dz is not None or dh is not None:
        dz = np.zeros(x.shape) if dz is None else np.asarray(dz, np.float64)
        dh = np.zeros(x.shape) if dh is None else np.asarray(dh, np.float64)
        u = dz * c
        dx = dh + r * (u - h * r ** 2 * (u * h).mean(1, keepdims=True))
        dt = dx * a
        out["dx"] = dx
        out["dy"] = ry * (dt - y * ry ** 2 * (dt * y).mean(1, keepdims=True)) if post else dt
        for name, table, each in (("dalpha", alpha, dx * t), ("dgamma", gamma, dz * h * r)):
            out[name] = None if table is None else by_group(each, group, np.asarray(table).size // d)
    return out


def by_group(each, group, groups):
    out = np.zeros((groups, each.shape[1]))
    for r in range(len(each)):
        g = 0 if group is None else int(group[r])
        if 0 <= g < groups:
            out[g] += each[r]
    return out


def grad_norm(grads, max_norm=None):
    """(norm, scale) of a list of gradients."""
    norm = np.sqrt(sum((np.asarray(g, np.float64) ** 2).sum() for g in grads))
    return norm, 1.0 if max_norm is None or norm <= max_norm else max_norm / norm
