"""Sums of attention weights and eviction by them from their definitions, in 64 bits on the CPU (numpy).

Error of a sum, derived from the number formats.  A weight is p = 2^(y - m) / l.  The logit y (in units of log2): products exact, their sum of dim terms off by at most
(dim + 8) 2^-24 sum |q_d k_d| scale, the further float operations by 2^-21 (|y| + 8), as in states_reference; with e the largest such error of the row, a weight is off by
2 e p, by the exponential's and the quotient's roundings (2^-21 p), by that of its divisor, a sum of n floats, 2 n 2^-24 p, and by 2^-126 where it is below the normal floats.
Sums of R weights in float, and with what was there before: (R + 2) 2^-24 of their size."""
import numpy as np

import states_reference as R


def weights(st, q, tables, lengths, q_start, scale, before=None):
    """(sums, allowed error) [sequences, heads, width * page] of attend_weights; st: an 8-bit store, or what states4_reference.held gives."""
    a, P = R.store_arrays(st), st.page_size
    tables = np.asarray(tables)
    S, width = tables.shape
    H, G, D = st.heads, q.shape[1] // st.heads, st.dim
    qn = q.detach().cpu().double().numpy().reshape(q.shape[0], H, G, D)
    out = np.zeros((S, H, width * P)) if before is None else np.asarray(before, np.float64).copy()
    tol = 2.0 ** -23 * np.abs(out)
    with np.errstate(all="ignore"):
        for s in range(S):
            lo, hi = int(q_start[s]), int(q_start[s + 1])
            length = min(max(int(lengths[s]), 0), width * P)
            t, (kc, _, ks, _) = R.gather(a, tables[s], P, st.pages, length)
            for h in range(H):
                k = kc[:, h] * ks[:, h, None]
                add, err = np.zeros(len(t)), np.zeros(len(t))
                for i in range(hi - lo):
                    seen = t <= length - (hi - lo) + i
                    if not seen.any():
                        continue
                    for g in range(G):
                        x = qn[lo + i, h, g]
                        z = scale * (k[seen] @ x)
                        p = np.exp(z - np.nanmax(z)) if not np.isnan(z).any() else np.full_like(z, np.nan)
                        p = p / p.sum()
                        e = (D + 8) * 2.0 ** -24 * abs(scale) * (np.abs(k[seen]) @ np.abs(x)).max() + 2.0 ** -21 * (np.abs(z).max() / np.log(2) + 8)
                        add[seen] += p
                        err[seen] += (2 * e + 2.0 ** -21 + 2 * seen.sum() * 2.0 ** -24) * p + 2.0 ** -126
                rows = (hi - lo) * G
                tol[s, h, t] += err + (rows + 2) * 2.0 ** -24 * (np.abs(out[s, h, t]) + add)
                out[s, h, t] += add
    return out, tol


def choose(sums, there, n, budget, recent):
    """Numbers of the kept keys of one sequence and head, in order.  sums [keys] float32, there [keys] bool."""
    keys = [j for j in range(n) if there[j]]
    if len(keys) <= budget:
        return keys
    new = [j for j in keys if j >= n - recent]
    old = [j for j in keys if j < n - recent]
    rank = lambda j: (0, -float(sums[j]), j) if not np.isnan(sums[j]) else (1, 0.0, j)  # noqa: E731
    return sorted(sorted(old, key=rank)[:budget - len(new)] + new)
