"""Definitions of the operators around a stage's linear layers, in fp64 and written for reading:
attention over packed sequences, the norms, the embedding, the distillation loss.

Plain numpy, one row or one sequence and head at a time.  Shares no code with the library."""
import numpy as np


def _f64(a):
    return np.asarray(a, dtype=np.float64)


# ---------------------------------------------------------------------------------------------
# attention: q [T, hq, d], k and v [T, hkv, d]; sequence s has the tokens starts[s] .. starts[s + 1] - 1
# ---------------------------------------------------------------------------------------------
def attention_forward(starts, q, k, v, scale):
    """(o [T, hq, d], lse [T, hq]).  Each query sees the keys of its sequence up to itself; a token of no
    sequence has o = 0 and lse = -infinity."""
    q, k, v = _f64(q), _f64(k), _f64(v)
    T, hq, _ = q.shape
    group = hq // k.shape[1]
    o, lse = np.zeros((T, hq, v.shape[2])), np.full((T, hq), -np.inf)
    for a, b in zip(starts[:-1], starts[1:]):
        for h in range(hq):
            for i in range(a, b):
                s = scale * (k[a:i + 1, h // group] @ q[i, h])
                m = s.max()
                e = np.exp(s - m)
                lse[i, h] = m + np.log(e.sum()) if m > -np.inf else m      # (nothing but -infinity: no result)
                o[i, h] = (e / e.sum()) @ v[a:i + 1, h // group]
    return o, lse


def attention_backward(starts, q, k, v, do, scale):
    """(dq, dk, dv) of sum(o * do)."""
    q, k, v, do = _f64(q), _f64(k), _f64(v), _f64(do)
    hq = q.shape[1]
    group = hq // k.shape[1]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for a, b in zip(starts[:-1], starts[1:]):
        for h in range(hq):
            g = h // group
            for i in range(a, b):
                K, V = k[a:i + 1, g], v[a:i + 1, g]
                s = scale * (K @ q[i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                dp = V @ do[i, h]
                ds = scale * p * (dp - p @ dp)
                dq[i, h] = ds @ K
                dk[a:i + 1, g] += np.outer(ds, q[i, h])
                dv[a:i + 1, g] += np.outer(p, do[i, h])
    return dq, dk, dv


# ---------------------------------------------------------------------------------------------
# norms of the rows of x [T, d]
# ---------------------------------------------------------------------------------------------
def norm_forward(x, weight, bias, eps, center):
    """(y, mean, rstd)."""
    x = _f64(x)
    mean = x.mean(1) if center else np.zeros(len(x))
    xc = x - mean[:, None]
    rstd = 1 / np.sqrt((xc ** 2).mean(1) + eps)
    return xc * rstd[:, None] * _f64(weight) + (0 if bias is None else _f64(bias)), mean, rstd


def norm_backward(x, weight, dy, eps, center):
    """(dx, dweight, dbias) of sum(y * dy)."""
    x, w, dy = _f64(x), _f64(weight), _f64(dy)
    _, mean, rstd = norm_forward(x, w, None, eps, center)
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * w
    dx = g - xh * (g * xh).mean(1, keepdims=True)
    if center:
        dx = dx - g.mean(1, keepdims=True)
    return dx * rstd[:, None], (dy * xh).sum(0), dy.sum(0)


# ---------------------------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------------------------
def embedding_forward(ids, table, scale):
    table = _f64(table)
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < len(table):
            out[t] = scale * table[i]
    return out


def embedding_backward(ids, dout, scale, n_rows):
    dout = _f64(dout)
    d = np.zeros((n_rows, dout.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < n_rows:
            d[i] += scale * dout[t]
    return d


# ---------------------------------------------------------------------------------------------
# distillation from a teacher's top logits
# ---------------------------------------------------------------------------------------------
def distill_loss(logits, ids, teacher, weight, temperature, grad_scale):
    """(loss [T], dlogits [T, V]): dlogits is the gradient of grad_scale * sum(loss)."""
    z, teacher = _f64(logits), _f64(teacher)
    T, V = z.shape
    loss, dz = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        w = 1.0 if weight is None else float(weight[t])
        named = [(int(i), x / temperature) for i, x in zip(ids[t], teacher[t]) if 0 <= i < V and x > -np.inf]
        if w == 0 or not named:
            continue
        x = np.array([v for _, v in named])
        logp = x - x.max()
        logp -= np.log(np.exp(logp).sum())
        y = z[t] / temperature
        logq = y - y.max()
        logq = logq - np.log(np.exp(logq).sum())
        g = np.exp(logq)
        for (i, _), lp in zip(named, logp):
            loss[t] += np.exp(lp) * (lp - logq[i])
            g[i] -= np.exp(lp)
        loss[t] *= w * temperature ** 2
        dz[t] = grad_scale * w * temperature * g
    return loss, dz
