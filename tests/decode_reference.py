"""The operators that decode over a cache, from their definitions in 64 bits (numpy, one sequence and head at a time),
and the error bounds that the kernels' arithmetic allows.

Bounds (u = 2^-24, half a step of fp32; b = 2^-8, half a step of bf16).  A score is a sum of D products of exactly
widened inputs in fp32, whatever the order: |error| <= (D + 2) u scale sum_d |q_d k_d|; call the largest over a row's keys
e_s.  The exponent's argument (score in units of log 2 minus maximum or log-sum-exp) takes up to 4 more roundings
of numbers no larger than X = max|score| + |lse|; ex2 is off by 2 units in the last place: so a weight is off by the
factor 1 +- e_p, e_p = e_s + 8 u X + 8 u (first order; the tests multiply bounds by 1.1).  Sums of n weights in fp32
add n u.
  out  |error| <= (2 e_p + 2 n u) A + c b A + b |out|, A = sum_j p_j |v_j| / sum_j p_j.  The last two terms are those of
       bf16: the result's rounding, and c = 1 where weights are rounded to bf16 before they multiply values.
  lse  |error| <= e_p + n u + 2 u X
  mass |error| <= sum_r w_r p_r (e_p + rows u) + 2 u |decay mass|
"""
import numpy as np

U, B16 = 2.0 ** -24, 2.0 ** -8


def sees_matrix(n, tree):
    """[n, n] truth values: node i sees node j.  tree: None (0 .. i) or int32 [n, words]."""
    if tree is None:
        return np.tri(n, dtype=bool)
    bits = np.unpackbits(np.ascontiguousarray(tree).view(np.uint8), axis=1, bitorder="little").astype(bool)
    full = np.zeros((n, n), bool)
    full[:, :min(n, bits.shape[1])] = bits[:, :n]
    return full


def attention(q, k, v, begin, length, offsets, dk, dv, tree, scale, bf16):
    """q [N, HQ, D], k, v [H, T, D], dk, dv [N, H, D] or None; float64 arrays.  Returns out, lse and their bounds (NaN
    in rows that belong to no sequence)."""
    N, HQ, D = q.shape
    H = k.shape[0]
    G = HQ // H
    out, lse = np.full(q.shape, np.nan), np.full((N, HQ), np.nan)
    out_tol, lse_tol = np.zeros(q.shape), np.zeros((N, HQ))
    for b in range(len(begin)):
        r, t = slice(begin[b], begin[b] + length[b]), slice(offsets[b], offsets[b + 1])
        n = offsets[b + 1] - offsets[b]
        sees = None if dk is None else sees_matrix(n, None if tree is None else tree[t])
        for x in range(HQ):
            for i in range(n):
                node = offsets[b] + i
                kk, vv = k[x // G, r], v[x // G, r]
                if dk is not None:
                    kk = np.concatenate([kk, dk[t][sees[i], x // G]])
                    vv = np.concatenate([vv, dv[t][sees[i], x // G]])
                m = len(kk)
                if m == 0:
                    out[node, x], lse[node, x] = 0, -np.inf
                    continue
                s = scale * (kk @ q[node, x])
                top = s.max()
                p = np.exp(s - top)
                l = p.sum()
                out[node, x], lse[node, x] = p @ vv / l, top + np.log(l)
                e_s = (D + 2) * U * scale * (np.abs(kk) @ np.abs(q[node, x])).max()
                X = np.abs(s).max() + abs(lse[node, x])
                e_p = e_s + 8 * U * X + 8 * U
                A = p @ np.abs(vv) / l
                out_tol[node, x] = (2 * e_p + 2 * m * U) * A + (B16 * A + B16 * np.abs(out[node, x]) if bf16 else U * np.abs(out[node, x]))
                lse_tol[node, x] = e_p + m * U + 2 * U * X
    return out, lse, 1.1 * out_tol, 1.1 * lse_tol


def attention_mass(q, lse, k, begin, length, offsets, scale, weight, decay, mass, rows):
    """Returns the collected weights [rows] (NaN outside the sequences) and their bounds."""
    N, HQ, D = q.shape
    H = k.shape[0]
    G = HQ // H
    got, tol = np.full(rows, np.nan), np.zeros(rows)
    for b in range(len(begin)):
        r = slice(begin[b], begin[b] + length[b])
        total, off = np.zeros(length[b]), np.zeros(length[b])
        n_rows = (offsets[b + 1] - offsets[b]) * HQ
        for node in range(offsets[b], offsets[b + 1]):
            w = 1.0 if weight is None else weight[node]
            if w == 0:
                continue
            for x in range(HQ):
                if lse[node, x] == -np.inf:
                    continue
                kk = k[x // G, r]
                s = scale * (kk @ q[node, x])
                p = w * np.exp(s - lse[node, x])
                e_p = (D + 2) * U * scale * (np.abs(kk) @ np.abs(q[node, x])) + 8 * U * (np.abs(s) + abs(lse[node, x])) + 8 * U
                total += p
                off += np.abs(p) * (e_p + (n_rows + 4) * U)
        old = 0.0 if mass is None or decay == 0 else decay * mass[r]
        got[r] = total + old
        tol[r] = off + 2 * U * np.abs(got[r]) + 2 * U * np.abs(old)
    return got, 1.1 * tol


def evict(mass, begin, length, budget, sink, recent):
    """kept rows (sequence by sequence) and offsets, by sorting."""
    kept, offsets = [], [0]
    for b in range(len(begin)):
        n = length[b]
        i = np.arange(n)
        x = mass[begin[b]:begin[b] + n].astype(np.float64) + 0.0
        second = ~((i < sink) | (i >= n - recent))
        nan = np.isnan(x)
        order = np.lexsort((i, np.where(nan, 0.0, -np.where(nan, 0.0, x)), ~nan, second))
        rows = np.sort(order[:max(0, min(budget[b], n))]) + begin[b]
        kept.append(rows)
        offsets.append(offsets[-1] + len(rows))
    return np.concatenate(kept).astype(np.int64) if kept else np.zeros(0, np.int64), np.asarray(offsets)
