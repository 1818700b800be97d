"""CPU oracle of what a recurrent language model's training has around its LSTM layers (test infrastructure, numpy float64): the gated
linear recurrence, label scores, the clipped AdamW step.

Definitions (time-major, masks as in lstm_oracle.py: frame t of row b is valid iff t < seq_lens[b]):

  gated scan    z = f | g | o pre-activations;  c_t = f c_{t-1} + (1 - f) tanh(z_g),  y = sigmoid(z_o) c_t,  f = sigmoid(z_f);
                padded frames carry c, give y = 0 and get dz = 0; direction -1 walks t = T-1 .. 0
  label score   lse, logp = x[label] - lse, entropy of the softmax, the best labels (larger value first, then smaller index), and the
                gradient of sum(dlogp logp) + sum(dent entropy); padded rows are 0 and have no alternatives
  AdamW         decoupled weight decay, bias corrections; 8-bit states: blocks of 256, values of 4 exponent and 3 mantissa bits times a
                scale per block, of m and of sqrt(v)
"""
import numpy as np


def _lens(seq_lens, T, B):
    return np.full(B, T) if seq_lens is None else np.clip(np.asarray(seq_lens), 0, T)


def _sig(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def gated_scan_fwd(z, c0=None, seq_lens=None, direction=1):
    """-> y [T, B, n], cT [B, n], before [T, B, n] (the state entering every frame)."""
    z = np.asarray(z, dtype=np.float64)
    T, B, n = z.shape[0], z.shape[1], z.shape[2] // 3
    L = _lens(seq_lens, T, B)
    c = np.zeros((B, n)) if c0 is None else np.array(c0, dtype=np.float64)
    y, before = np.zeros((T, B, n)), np.zeros((T, B, n))
    for t in (range(T) if direction > 0 else range(T - 1, -1, -1)):
        before[t] = c
        ok = t < L
        zt = z[t, ok]
        c = c.copy()
        c[ok] = _sig(zt[:, :n]) * c[ok] + _sig(-zt[:, :n]) * np.tanh(zt[:, n:2 * n])
        y[t, ok] = _sig(zt[:, 2 * n:]) * c[ok]
    return y, c, before


def gated_scan_bwd(z, dy, c0=None, seq_lens=None, dcT=None, direction=1):
    """-> dz [T, B, 3n], dc0 [B, n], db [3n]."""
    z, dy = np.asarray(z, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    T, B, n = z.shape[0], z.shape[1], z.shape[2] // 3
    L = _lens(seq_lens, T, B)
    before = gated_scan_fwd(z, c0, seq_lens, direction)[2]
    dz, e = np.zeros_like(z), np.zeros((B, n)) if dcT is None else np.array(dcT, dtype=np.float64)
    for t in (range(T - 1, -1, -1) if direction > 0 else range(T)):
        ok = t < L
        zt, cp, d = z[t, ok], before[t, ok], dy[t, ok]
        f, nf, g, o, no = _sig(zt[:, :n]), _sig(-zt[:, :n]), np.tanh(zt[:, n:2 * n]), _sig(zt[:, 2 * n:]), _sig(-zt[:, 2 * n:])
        dc = d * o + e[ok]
        dz[t, ok] = np.concatenate([dc * (cp - g) * f * nf, dc * nf * (1 - g * g), d * (f * cp + nf * g) * o * no], axis=1)
        e[ok] = f * dc
    return dz, e, dz.sum(axis=(0, 1))


def label_score_fwd(x, label=None, seq_lens=None, top=0):
    """x [T, B, V] -> dict(logp, entropy, lse [T, B], q = log p [T, B, V], top_logp, top_label [T, B, top]).  Differences of logits are
    taken from the maximum: lse itself has no digits left for log z where the logits are as large as a float allows."""
    x = np.asarray(x, dtype=np.float64)
    T, B, V = x.shape
    L = _lens(seq_lens, T, B)
    out = dict(logp=np.zeros((T, B)), entropy=np.zeros((T, B)), lse=np.zeros((T, B)), q=np.zeros(x.shape), top_logp=np.full((T, B, top), -np.inf), top_label=np.zeros((T, B, top), dtype=np.int64))
    for t in range(T):
        for b in range(B):
            if t >= L[b]:
                continue
            r, l = x[t, b], None if label is None else int(label[t, b])
            if np.isnan(r).any() or (r == np.inf).any():
                out["lse"][t, b] = out["entropy"][t, b] = out["q"][t, b] = np.nan
                out["logp"][t, b] = np.nan if l is not None and 0 <= l < V else 0
                continue
            m = r.max()
            if m == -np.inf:
                out["lse"][t, b] = -np.inf
                out["logp"][t, b] = -np.inf if l is not None and 0 <= l < V else 0
                continue
            e = np.exp(r - m)
            p, q = e / e.sum(), (r - m) - np.log(e.sum())
            out["lse"][t, b], out["q"][t, b] = m + np.log(e.sum()), q
            out["entropy"][t, b] = -(p[p > 0] * q[p > 0]).sum()
            if l is not None and 0 <= l < V:
                out["logp"][t, b] = q[l]
            order = np.lexsort((np.arange(V), -r))[:top]
            order = order[r[order] > -np.inf]
            out["top_logp"][t, b, :len(order)] = q[order]
            out["top_label"][t, b, :len(order)] = order
    return out


def label_score_bwd(x, label, dlogp, dent=None, seq_lens=None):
    """-> dlogits [T, B, V]."""
    x = np.asarray(x, dtype=np.float64)
    T, B, V = x.shape
    L, f, d = _lens(seq_lens, T, B), label_score_fwd(x, label, seq_lens), np.zeros(x.shape)
    for t in range(T):
        for b in range(B):
            l = -1 if label is None else int(label[t, b])
            wl, we = dlogp[t, b] if dlogp is not None and 0 <= l < V else 0.0, 0.0 if dent is None else dent[t, b]
            if t >= L[b] or (wl == 0 and we == 0) or f["lse"][t, b] == -np.inf:
                continue
            q = f["q"][t, b]
            p = np.exp(q)
            d[t, b] = -wl * p - we * p * (np.where(p > 0, q, 0) + f["entropy"][t, b])         # (lse is NaN: so is all of it)
            if wl:
                d[t, b, l] += wl
    return d


BLOCK = 256


def values8():
    """The non-negative finite e4m3 values, in the order of their codes 0 .. 126."""
    code = np.arange(127)
    e, m = code >> 3, code & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


def to8(x):
    """Magnitudes up to 448 -> the nearest value (ties to the even code), sign kept."""
    x = np.asarray(x, dtype=np.float64)
    v, a = values8(), np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(v, a), 1, 126)
    lo = hi - 1
    up = (a - v[lo] > v[hi] - a) | ((a - v[lo] == v[hi] - a) & (hi % 2 == 0))
    return np.copysign(np.where(up, v[hi], v[lo]), x)


def spread(scale, n):
    return np.repeat(scale, BLOCK)[:n]


def block_scale(x):
    n = x.size
    return np.abs(np.pad(x, (0, -n % BLOCK))).reshape(-1, BLOCK).max(1) / 448.0 if n else np.zeros(0)


def adamw(w, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, scale=1.0):
    """-> w, m, v after the step; 8-bit states are the caller's business (m and v in their values)."""
    if not np.isfinite(scale):
        return w, m, v
    g = g * scale
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    w = w * (1 - lr * decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w, m, v


def grad_norm(grads, max_norm=np.inf):
    norm = np.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))
    return norm, (min(1.0, max_norm / norm) if norm > 0 else 1.0) if np.isfinite(norm) else np.nan
