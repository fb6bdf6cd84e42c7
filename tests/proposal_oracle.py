"""Plain 64-bit implementations of the 8-bit proposal path's definitions (numpy, CPU)."""
import math

import numpy as np

E4M3 = None  # the 127 non-negative finite values, code by code


def e4m3_values():
    global E4M3
    if E4M3 is None:
        c = np.arange(127)
        e, m = c >> 3, c & 7
        E4M3 = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    return E4M3


def decode(q):
    """Values of e4m3 codes (uint8); code 127 is NaN."""
    v = np.append(e4m3_values(), np.nan)[q & 127]
    return np.where(q & 128, -v, v)


def quantize(x, block_rows):
    """(codes uint8, scales float32) of x (float64 of fp32 or bf16 values)."""
    rows, cols = x.shape
    gr, gc = -(-rows // block_rows), -(-cols // 128)
    p = np.zeros((gr * block_rows, gc * 128))
    p[:rows, :cols] = x
    g = p.reshape(gr, block_rows, gc, 128)
    finite = np.isfinite(g).all(axis=(1, 3))
    top = np.where(finite, np.abs(np.where(np.isfinite(g), g, 0)).max(axis=(1, 3)), np.nan)
    scale = np.maximum(top / 448.0, 2.0 ** -126).astype(np.float32)
    v = g / scale.astype(np.float64)[:, None, :, None]
    a = np.abs(np.where(np.isnan(v), 0.0, v))
    values = e4m3_values()
    mid = (values[1:] + values[:-1]) / 2
    code = np.searchsorted(mid, a)  # a on a border: the lower code
    low = np.minimum(code, 125)
    code = np.where((code < 126) & (a == mid[low]) & (code % 2 == 1), code + 1, np.minimum(code, 126))
    code = code | np.where(np.signbit(g) & finite[:, None, :, None], 128, 0)
    return code.reshape(gr * block_rows, gc * 128)[:rows, :cols].astype(np.uint8), scale


def logits(h, hs, w, ws, bias):
    """(z, sum of magnitudes) from codes and scales, float64."""
    K = h.shape[1]
    rep = lambda s, n: np.repeat(s.astype(np.float64), 128, axis=1)[:, :n]  # noqa: E731
    hv = decode(h) * rep(hs, K)
    wv = decode(w) * np.repeat(rep(ws, K), 128, axis=0)[:w.shape[0]]
    z, mag = hv @ wv.T, np.abs(hv) @ np.abs(wv).T
    return (z if bias is None else z + bias), mag


def sample_row(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, kept, probs, logprob) of one row (z: any float type) by the definition."""
    V = len(z)
    z = z.astype(np.float64)
    ok = T >= 0 and math.isfinite(T) and 0 <= p <= 1 and 0 <= m <= 1 and 0 <= u < 1
    if not ok or np.isnan(z).any() or (z == np.inf).any() or not np.isfinite(z).any():
        return -1, 0, np.zeros(V), np.nan
    if T == 0:
        T, k = 1.0, 1
    order = np.argsort(-z, kind="stable")
    n = int(np.isfinite(z).sum())
    if 0 < k < n:
        n = k
    order = order[:n]
    w = np.exp((z[order] - z[order[0]]) / T)
    if p < 1:
        mass = np.cumsum(w)
        n = min(int(np.searchsorted(mass, p * mass[-1], side="left")) + 1, n)
    n = min(n, int((w[:n] >= m).sum()))
    order, w = order[:n], w[:n]
    by_id = np.argsort(order)
    mass = np.cumsum(w[by_id])
    at = int(np.searchsorted(mass, u * mass[-1], side="right"))
    probs = np.zeros(V)
    probs[order] = w / mass[-1]
    token = int(order[by_id[at]])
    x = (z[token] - z[order[0]]) / T
    return token, n, probs, x - math.log(mass[-1])
