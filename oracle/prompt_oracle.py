"""Plain 64-bit implementation of causal attention over packed sequences and its gradient (vla_prompt.h), one sequence and
head at a time, with the sums of magnitudes that error bounds need."""
import numpy as np


def sequences(row_start, rows):
    """(first row, rows) of the sequences whose bounds ascend within the tensors."""
    return [(a, b - a) for a, b in zip(row_start, row_start[1:]) if 0 <= a < b <= rows]


def weights(q, k, scale):
    """(causal softmax weights, log-sum-exp, largest sum of |q k| |scale|) of one head; q, k [n, head_dim]."""
    n = len(q)
    s = q @ k.T * scale
    s[np.triu_indices(n, 1)] = -np.inf
    m = s.max(1)
    m0 = np.where(np.isneginf(m), 0.0, m)
    e = np.exp(s - m0[:, None])
    z = e.sum(1)
    with np.errstate(divide="ignore"):
        lse = m0 + np.log(z)
    p = e / np.where(z == 0, 1.0, z)[:, None]
    return p, lse, (np.abs(q) @ np.abs(k).T * np.tri(n)).max(1) * abs(scale)


def attention(q, k, v, row_start, scale):
    """(out, lse, sum_j p_ij |v_j| as out, largest sum of |q k| |scale| as lse); rows of no sequence are NaN."""
    rows, H, hd = q.shape
    G = H // k.shape[1]
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, smax = np.full((rows, H), np.nan), np.full((rows, H), np.nan)
    for a, n in sequences(row_start, rows):
        r = slice(a, a + n)
        for h in range(H):
            p, lse[r, h], smax[r, h] = weights(q[r, h], k[r, h // G], scale)
            out[r, h] = p @ v[r, h // G]
            mag[r, h] = p @ np.abs(v[r, h // G])
    return out, lse, mag, smax


def backward(q, k, v, dout, row_start, scale, unit_w=0.0, unit_p=0.0, unit_dp=0.0, out_err=None):
    """(dq, dk, dv) and bounds of their errors, where every weight is off by a relative unit_w as it meets the other factor of
    its product, p itself by unit_p times the largest score's magnitude, dP and the sums by a relative unit_dp of their
    terms' magnitudes, and `out` by out_err [rows, heads, head_dim].  Rows of no sequence are NaN."""
    rows, H, hd = q.shape
    G = H // k.shape[1]
    g = [np.full(x.shape, np.nan) for x in (q, k, v)]
    e = [np.full(x.shape, np.nan) for x in (q, k, v)]
    for a, n in sequences(row_start, rows):
        r = slice(a, a + n)
        for x in (g[1], g[2], e[1], e[2]):
            x[r] = 0.0
        for h in range(H):
            kv = h // G
            Q, K, V, D = q[r, h], k[r, kv], v[r, kv], dout[r, h]
            p, _, smax = weights(Q, K, scale)
            dp, o = D @ V.T, p @ V
            ds = p * (dp - (D * o).sum(1)[:, None])
            g[0][r, h] = scale * ds @ K
            g[1][r, kv] += scale * ds.T @ Q
            g[2][r, kv] += p.T @ D
            ep = p * unit_p * np.maximum(smax, 1.0)[:, None]
            adp = np.abs(D) @ np.abs(V).T
            eD = unit_dp * (np.abs(D) * np.abs(o)).sum(1)
            if out_err is not None:
                eD = eD + (np.abs(D) * out_err[r, h]).sum(1)
            eds = np.abs(ds) * (unit_w + unit_dp * n) + ep * np.abs(dp - (D * o).sum(1)[:, None]) + p * (unit_dp * adp + eD[:, None])
            e[0][r, h] = abs(scale) * eds @ np.abs(K)
            e[1][r, kv] += abs(scale) * eds.T @ np.abs(Q)
            e[2][r, kv] += (ep + p * (unit_w + unit_dp * n)).T @ np.abs(D)
    return g, e
