"""The operators round a cache in 8 bits, from their definitions in 64 bits (numpy), and the error bounds that the kernels'
arithmetic allows.

Bounds, with u = 2^-24 (half a step of fp32) and h half a step of the storage type (2^-8 for bf16, u for fp32):
  norm and rotation   the mean of D squares is off by (D + 2) u, so 1 / sqrt by (D / 2 + 4) u with rsqrt's own two units in
      the last place, and y = x f w by (D / 2 + 7) u |y|.  An angle is a fraction of a turn rounded to fp32 (pi u) with the
      error of its formation in 64 bits, 2^-52 |angle|, and sine and cosine are off by two units: 8 u + 2^-51 |angle| in all.  Two products
      and their sum: 2 u.  |error| <= ((D / 2 + 17) u + 2^-51 |angle|) (|y_i| + |y_j|) + h |out|.
  codes and scales    none: a scale is a power of two chosen by comparison, multiplying by it is exact, and the nearest code
      is a matter of the value alone.
  attention           as in decode_reference, over the values that the codes stand for.  The values' exponents (up to E) are added to
      the scores, and taken out of the sum again: X = max |score| + |lse| + E.  Query rows in fp16: a product is off by 2^-39 of the
      row's largest element times the code's value.  Weights are rounded to bf16 or finer; in fp16 the largest (times its scale) is
      2^8 at least, and those under 2^-14 are off by half a step of 2^-24, 2^-33 of it: n 2^-33 448 max_j p_j 2^e_j / l.
"""
import numpy as np

from decode_reference import B16, U, sees_matrix

TOP = {"e4m3": 448.0, "i8": 127.0}
LEAST, MOST = -48, 48


def e4m3_values():
    """Values of the 256 codes."""
    code = np.arange(256)
    e, m = code >> 3 & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(code & 127) == 127] = np.nan
    return np.where(code >= 128, -v, v)


def values_of(codes, kind):
    """Values of codes (uint8 bits)."""
    return e4m3_values()[codes] if kind == "e4m3" else codes.view(np.int8).astype(np.float64)


def nearest(x, kind):
    """Codes (uint8 bits) nearest to x, ties to even, the largest beyond them; NaN: NaN, or 0."""
    x = np.asarray(x, np.float64)
    if kind == "i8":
        return np.where(np.isnan(x), 0, np.clip(np.rint(np.nan_to_num(x, nan=0.0)), -128, 127)).astype(np.int8).view(np.uint8)
    table = e4m3_values()[:127]
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=1e9, neginf=-1e9)), 448.0)
    lo = np.clip(np.searchsorted(table, a, side="right") - 1, 0, 125)
    mid = (table[lo] + table[lo + 1]) / 2
    code = np.where((a > mid) | ((a == mid) & (lo % 2 == 1)), lo + 1, lo)
    code = np.where(np.isnan(x), 127, code | np.where(np.signbit(x), 128, 0))
    return code.astype(np.uint8)


def exponent(top, kind):
    if top == 0:
        return LEAST
    e = int(np.ceil(np.log2(top / TOP[kind])))
    while top > TOP[kind] * 2.0 ** e:
        e += 1
    while top <= TOP[kind] * 2.0 ** (e - 1):
        e -= 1
    return min(max(e, LEAST), MOST)


def clamped(scales):
    return np.clip(scales.astype(int) - 127, LEAST, MOST)


def append(x, codes, scales, kind, block, to):
    """Plane by plane: rows x [n, D] (float64) go to rows to .. to + n - 1 of codes [T, D] (uint8), scales [blocks], in place."""
    n = len(x)
    for blk in range(to // block, (to + n - 1) // block + 1):
        r0, r1 = max(to, blk * block), min(to + n, (blk + 1) * block)
        mine = x[r0 - to:r1 - to]
        finite = np.abs(mine[np.isfinite(mine)])
        e = exponent(finite.max(initial=0.0), kind)
        if r0 > blk * block:
            old = clamped(scales[blk])
            e = max(e, int(old))
            front = codes[blk * block:r0]
            if e != old:
                codes[blk * block:r0] = nearest(values_of(front, kind) * 2.0 ** (old - e), kind)
        scales[blk] = e + 127
        codes[r0:r1] = nearest(mine * 2.0 ** -e, kind)


def norm_rope(x, positions, axis, base, weight, eps, norm, half_step):
    """x [N, heads, D] float64; returns out and its bound."""
    D, half = x.shape[2], len(axis)
    y = x
    if norm:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else weight)
    out, near = y.copy(), np.abs(y)
    if half:
        angle = positions[axis].T.astype(np.float64) * base ** (-np.arange(half) / half)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        a, b = y[..., :half], y[..., half:2 * half]
        out[..., :half], out[..., half:2 * half] = a * c - b * s, b * c + a * s
        both = (np.abs(a) + np.abs(b)) * (1 + 2.0 ** -51 * np.abs(angle)[:, None] / ((D / 2 + 17) * U))
        near[..., :half] = near[..., half:2 * half] = both
    return out, 1.1 * ((D / 2 + 17) * U * near + half_step * np.abs(out))


def attention(q, kc, ks, vc, vs, kind, block, begin, length, offsets, dk, dv, tree, scale):
    """q [N, HQ, D], codes kc, vc [H, T, D] (uint8), scales ks, vs [H, blocks], dk, dv [N, H, D] or None; returns out, lse and
    their bounds."""
    N, HQ, D = q.shape
    G = HQ // kc.shape[0]
    out, lse = np.full(q.shape, np.nan), np.full((N, HQ), np.nan)
    out_tol, lse_tol = np.zeros(q.shape), np.zeros((N, HQ))
    for b in range(len(begin)):
        rows = np.arange(begin[b], begin[b] + length[b])
        t = slice(offsets[b], offsets[b + 1])
        n = offsets[b + 1] - offsets[b]
        sees = None if dk is None else sees_matrix(n, None if tree is None else tree[t])
        for h in range(kc.shape[0]):
            ke, ve = clamped(ks[h, rows // block]), clamped(vs[h, rows // block])
            k8 = values_of(kc[h, rows], kind) * 2.0 ** ke[:, None]
            v8 = values_of(vc[h, rows], kind) * 2.0 ** ve[:, None]
            for x in range(h * G, (h + 1) * G):
                for i in range(n):
                    node = offsets[b] + i
                    kk, vv, ee = k8, v8, ve
                    if dk is not None:
                        kk = np.concatenate([kk, dk[t][sees[i], h]])
                        vv = np.concatenate([vv, dv[t][sees[i], h]])
                        ee = np.concatenate([ee, np.zeros(sees[i].sum(), int)])
                    m = len(kk)
                    if m == 0:
                        out[node, x], lse[node, x] = 0, -np.inf
                        continue
                    s = scale * (kk @ q[node, x])
                    top = s.max()
                    p = np.exp(s - top)
                    l = p.sum()
                    out[node, x], lse[node, x] = p @ vv / l, top + np.log(l)
                    size = np.abs(kk).sum(1).max()
                    e_s = (D + 2) * U * scale * (np.abs(kk) @ np.abs(q[node, x])).max() + scale * 2.0 ** -39 * np.abs(q[node, x]).max() * size
                    X = np.abs(s).max() + abs(lse[node, x]) + np.abs(ee).max()
                    e_p = e_s + 8 * U * X + 8 * U
                    A = p @ np.abs(vv) / l
                    low = m * 2.0 ** -33 * 448 * (p * 2.0 ** ee).max() / l
                    out_tol[node, x] = (2 * e_p + 2 * m * U) * A + B16 * A + B16 * np.abs(out[node, x]) + low
                    lse_tol[node, x] = e_p + m * U + 2 * U * X
    return out, lse, 1.1 * out_tol, 1.1 * lse_tol
