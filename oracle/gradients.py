"""Gradients for the optimizer steps, in binary64: embedding lookup and gradient, 8-bit activation checkpoints, the gated
activation's and the linear layers' backward passes from them.  Plain loops over the definitions; no GPU code."""
import numpy as np

GROUP = 32


def embed_lookup(table, ids, scale, pad_id=None):
    """x_i = scale * table[id_i], zero at padding and for ids outside the table."""
    out = np.zeros((len(ids), table.shape[1]))
    for t, v in enumerate(ids):
        if (pad_id is None or v != pad_id) and 0 <= v < table.shape[0]:
            out[t] = scale * table[v]
    return out


def embed_grad(dx, ids, vocab, scale, pad_id=None, start=None):
    """G[v] = (start[v] +) scale * sum of dx_i over id_i = v; padding and ids outside the table add nothing."""
    out = np.zeros((vocab, dx.shape[1]))
    for t, v in enumerate(ids):
        if (pad_id is None or v != pad_id) and 0 <= v < vocab:
            out[v] += dx[t]
    out *= scale
    return out if start is None else start + out


def ckpt_pack(x):
    """(q, e) of a rows x cols matrix: per group of 32 columns the least k >= -126 with max|x| <= 127 * 2^k,
    q = x / 2^k rounded half to even (held at 63 for k = 122, where 64 stands for an infinity), e = k + 127; e = 255
    and q = 0 for a group with a NaN or an infinity."""
    rows, cols = x.shape
    ld = -(-cols // GROUP) * GROUP
    q = np.zeros((rows, ld), dtype=np.int8)
    e = np.zeros((rows, ld // GROUP), dtype=np.uint8)
    for r in range(rows):
        for g in range(ld // GROUP):
            v = x[r, g * GROUP:(g + 1) * GROUP]
            if not np.isfinite(v).all():
                e[r, g] = 255
                continue
            top, k = np.abs(v).max(), -126
            while top > 127.0 * 2.0 ** k:
                k += 1
            e[r, g] = k + 127
            q[r, g * GROUP:g * GROUP + len(v)] = np.clip(np.rint(v / 2.0 ** k), *((-63, 63) if k == 122 else (-127, 127)))
    return q, e


def ckpt_values(q, e, cols):
    """q * 2^(e - 127); NaN where e = 255."""
    scale = np.where(e == 255, np.nan, 2.0 ** (e.astype(np.float64) - 127.0))
    return (q.astype(np.float64) * np.repeat(scale, GROUP, axis=1))[:, :cols]


def gate_forward(g, u):
    """h = silu(g) * u."""
    return g / (1.0 + np.exp(-g)) * u


def gate_grad(g, u, dh):
    """(dgate, dup) of h = silu(g) * u."""
    s = 1.0 / (1.0 + np.exp(-g))
    return dh * u * s * (1.0 + g * (1.0 - s)), dh * g * s


def weight_grad(dy, x, start=None):
    """G = (start +) sum over tokens of dy_t x_t^T."""
    out = dy.T @ x
    return out if start is None else start + out
