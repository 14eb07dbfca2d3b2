"""float64 CPU oracle for the operators of finetuning a pruned student: attention with a
learned relative position bias and its gradients, and the distillation loss from a
teacher's top logits with its gradient.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  Written as the definitions in
float64 numpy, one sequence and head (or one row) at a time.
"""
import numpy as np


def _pairs(index, region, lowest, bias):
    """The T x T truth values of the pairs that take part."""
    ok = (index >= 0) & (bias > lowest)
    if region is not None:
        ok &= (region[:, None] == region[None, :]) & (region[:, None] >= 0)
    return ok


def relpos_attention(qkv, table, index, n_seq, H, hd, region=None, dout=None, lowest=-np.inf):
    """Attention of n_seq sequences of T = len(index) tokens with the bias
    table[index[i, j], h] (index -1, a bias at or below ``lowest``, labels that differ or are
    negative: no pair).  Returns a dict of out, lse and, with dout, dqkv and dtable, plus
    the sums of absolute values that rounding bounds are made of."""
    T = index.shape[0]
    x = np.asarray(qkv, np.float64).reshape(n_seq, T, 3, H, hd)
    r = {"out": np.zeros((n_seq, T, H, hd)), "lse": np.full((n_seq, H, T), -np.inf),
         "abs_pv": np.zeros((n_seq, T, H, hd)), "abs_s": np.zeros((n_seq, H, T))}
    if dout is not None:
        g = np.asarray(dout, np.float64).reshape(n_seq, T, H, hd)
        r.update(dqkv=np.zeros((n_seq, T, 3, H, hd)), dtable=np.zeros(table.shape),
                 P=np.zeros((n_seq, H, T, T)), dP=np.zeros((n_seq, H, T, T)),
                 abs_dP=np.zeros((n_seq, H, T, T)), D=np.zeros((n_seq, H, T)))
    at = np.clip(index, 0, None)
    for n in range(n_seq):
        lab = None if region is None else region[n % len(region)]
        pad = np.zeros(T, bool) if lab is None else lab < 0
        for h in range(H):
            q, k, v = (np.where(pad[:, None], 0.0, x[n, :, i, h]) for i in range(3))
            b = table[at, h].astype(np.float64)
            ok = _pairs(index, lab, lowest, b)
            s = np.where(ok, (q @ k.T) / np.sqrt(hd) + np.where(ok, b, 0.0), -np.inf)
            some = ok.any(1)
            m = np.where(some, s.max(1), 0.0)
            e = np.exp(s - m[:, None])
            total = e.sum(1)
            p = e / np.where(some, total, 1.0)[:, None]
            r["lse"][n, h, some] = (m + np.log(np.where(some, total, 1.0)))[some]
            r["out"][n, :, h] = p @ v
            r["abs_pv"][n, :, h] = p @ np.abs(v)
            r["abs_s"][n, h] = np.where(ok, np.abs(q) @ np.abs(k).T / np.sqrt(hd) +
                                        np.where(ok, np.abs(b), 0.0), 0.0).max(1)
            if dout is None:
                continue
            do = np.where(pad[:, None], 0.0, g[n, :, h])
            dp = do @ v.T
            D = (p * dp).sum(1)
            ds = p * (dp - D[:, None])
            r["dqkv"][n, :, 0, h] = ds @ k / np.sqrt(hd)
            r["dqkv"][n, :, 1, h] = ds.T @ q / np.sqrt(hd)
            r["dqkv"][n, :, 2, h] = p.T @ do
            np.add.at(r["dtable"][:, h], at[ok], ds[ok])
            r["P"][n, h], r["dP"][n, h], r["D"][n, h] = p, dp, D
            r["abs_dP"][n, h] = np.abs(do) @ np.abs(v).T
    for key, cols in (("out", H * hd), ("abs_pv", H * hd), ("dqkv", 3 * H * hd)):
        if key in r:
            r[key] = r[key].reshape(n_seq * T, cols)
    return r


def distill(logits, ids, teacher, temperature, dloss=None):
    """loss = t^2 sum_j q_j (log q_j - log p[id_j]) per row, p = softmax(logits / t), q the
    softmax of teacher / t over the row's entries with an id in [0, V) (and a logit above
    -inf); 0 for a row without any.  With dloss, also dlogits = dloss t (p - the q of each class)."""
    z = np.asarray(logits, np.float64) / temperature
    M, V = z.shape
    loss, grad = np.zeros(M), np.zeros((M, V))
    for r in range(M):
        use = np.flatnonzero((ids[r] >= 0) & (ids[r] < V) & (teacher[r] > -np.inf))
        if not len(use):
            continue
        at, t = ids[r, use], np.asarray(teacher[r, use], np.float64) / temperature
        log_q = t - t.max() - np.log(np.exp(t - t.max()).sum())
        log_p = z[r] - z[r].max() - np.log(np.exp(z[r] - z[r].max()).sum())
        q = np.exp(log_q)
        have = q > 0
        loss[r] = temperature ** 2 * (q[have] * (log_q[have] - log_p[at[have]])).sum()
        if dloss is not None:
            d = np.exp(log_p)
            np.subtract.at(d, at, q)
            grad[r] = dloss[r] * temperature * d
    return (loss, grad) if dloss is not None else loss
