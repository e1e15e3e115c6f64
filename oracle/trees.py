"""Trees of candidates and verification by sampling, in float64 numpy.

A tree of k candidates is a list of parents (parents[i] < i, -1 the root);
row 0 is the root, row i + 1 candidate i.
"""
import numpy as np


def chain(k):
    return list(range(-1, k - 1))


def visible(parents):
    """[rows, rows] truth values: row i is or follows row j."""
    m = np.eye(len(parents) + 1, dtype=bool)
    for i, p in enumerate(parents):
        m[i + 1] |= m[p + 1]
    return m


def depths(parents):
    return (visible(parents).sum(1) - 1).tolist()


def attention(q, K, V, k, v, parents):
    """q [rows, n_q, d] over the cache K, V [keys, n_kv, d] and the tree's k, v [rows, n_kv, d]."""
    rows, n_q, d = q.shape
    n_kv, sees = K.shape[1], visible(parents)
    out = np.empty((rows, n_q, d))
    for i in range(rows):
        kk, vv = np.concatenate([K, k[sees[i]]]), np.concatenate([V, v[sees[i]]])
        for h in range(n_q):
            g = h * n_kv // n_q
            s = kk[:, g] @ q[i, h] / np.sqrt(d)
            p = np.exp(s - s.max())
            out[i, h] = p @ vv[:, g] / p.sum()
    return out


def greedy_walk(tokens, cands, parents):
    """Accepted candidates and the token after them, from the rows' greedy tokens."""
    node, path = -1, []
    while True:
        after = [i for i, p in enumerate(parents) if p == node and cands[i] == tokens[node + 1]]
        if not after:
            return path, int(tokens[node + 1])
        node = after[0]
        path.append(node)


def log_softmax(logits, temperature):
    z = np.asarray(logits, dtype=np.float64) / temperature
    z = z - z.max()
    return z - np.log(np.exp(z).sum())


def sample_walk(target, cands, uniforms, parents, temperature=1.0, draft=None, draft_temperature=None):
    """(path, token, logp): the candidates tested in order against what is
    left of the target's distribution at their node, then one token of it.
    target, draft: logits [rows, vocab]; uniforms: one per candidate, and one."""
    k = len(cands)
    lp = [log_softmax(row, temperature) for row in target]
    node, path, left = -1, [], np.exp(lp[0])
    for i in range(k):
        if parents[i] != node:
            continue
        x = int(cands[i])
        inside = 0 <= x < left.size
        mass = left.sum()
        if draft is None:
            q = np.zeros_like(left)
            if inside:
                q[x] = 1.0
        else:
            q = np.exp(log_softmax(draft[node + 1], draft_temperature or temperature))
        if inside and float(uniforms[i]) * mass * q[x] < left[x]:
            path.append(i)
            node, left = i, np.exp(lp[i + 1])
        elif draft is None:
            left = left.copy()
            if inside:
                left[x] = 0.0
        else:
            left = np.maximum(left - mass * q, 0.0)
    if not left.sum() > 0:
        left = np.exp(lp[node + 1])
    run = np.cumsum(left)
    token = int(np.argmax(run > float(uniforms[k]) * run[-1]))
    logp = [lp[p + 1][int(x)] if 0 <= int(x) < left.size else -np.inf for p, x in zip(parents, cands)]
    return path, token, logp + [lp[node + 1][token]]
