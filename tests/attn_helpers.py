"""Attention tests: device inputs with guarded surroundings, the binary64 oracle, and bounds on how far a result may be off.

Bounds.  Scores are dot products of d terms in binary32, off by at most (d + 8) 2^-24 (a + |L| + 1), a = scale sum |q k|: the
products' sum, the scale, the subtraction of a maximum or of L, and the exponential (an error of its own of 2^-23).  That is a
relative error `ep` of a probability.  The forward pass divides by a sum of them, which is off by the largest ep too and by
(m + 8) 2^-24 for m terms; bf16 adds half a step, 2^-8, for the rounding of each P (of P and of S in the gradient), and the
result its own rounding u.  dP - D is off by (d + 8) 2^-24 of its terms' magnitudes.  1 + 2^-5 covers the products of bounds.

dQ in bf16 is sum round(S_j) k_j + c sum (S_j - round(S_j)), c the mean of some keys that the query sees: off by
sum (S_j - round(S_j)) (k_j - c), at most 2^-8 sum |S_j| (|k_j| + max |k|), the maximum over the keys that the query sees."""
import numpy as np

from oracle import gradients as gr

import paper_2607_19331_amd as iso
from tests.grad_helpers import Mat, close, code, ttype, unit

E24 = 2.0 ** -24
SLACK = 1 + 2.0 ** -5


def f64(a, dtype):
    import torch
    return torch.as_tensor(np.ascontiguousarray(a)).to(ttype(dtype)).double().numpy()


class Case:
    """Packed sequences: `before` rows in front of the first one and 5 behind the last belong to none and hold NaN."""

    def __init__(self, dtype, lens_q, lens_k, heads, kv, dim, causal, window=0, gap=0, seed=0, before=2, edit=None, scale=None):
        import torch
        rng = np.random.default_rng(seed + 7 * dim + sum(lens_q))
        self.dtype, self.lens_q, self.lens_k, self.heads, self.kv, self.dim = dtype, lens_q, lens_k, heads, kv, dim
        self.causal, self.window, self.scale = causal, window, 1.0 / np.sqrt(dim) if scale is None else scale
        self.at_q = before + np.concatenate([[0], np.cumsum(lens_q)]).astype(np.int64)
        self.at_k = before + np.concatenate([[0], np.cumsum(lens_k)]).astype(np.int64)
        nq, nk = int(self.at_q[-1]) + 5, int(self.at_k[-1]) + 5
        bias = rng.standard_normal(kv * dim)
        self.host = {}
        for name, rows, cols, sigma in (("q", nq, heads * dim, 1.5), ("k", nk, kv * dim, 1.0), ("v", nk, kv * dim, 1.0),
                                        ("dout", nq, heads * dim, 0.1)):
            x = rng.standard_normal((rows, cols)) * sigma + (bias if name == "k" else 0.0)
            at = self.at_q if rows == nq and name in ("q", "dout") else self.at_k
            x[:at[0]] = np.nan
            x[at[-1]:] = np.nan
            self.host[name] = x
        if edit is not None:
            edit(self)
        self.host = {n: f64(x, dtype) for n, x in self.host.items()}
        mat = lambda n: Mat(*self.host[n].shape, dtype, gap, self.host[n])  # noqa: E731
        self.q, self.k, self.v, self.dout = (mat(n) for n in ("q", "k", "v", "dout"))
        self.out = Mat(nq, heads * dim, dtype, gap)
        self.dq, self.dk, self.dv = Mat(nq, heads * dim, dtype, gap), Mat(nk, kv * dim, dtype, gap), Mat(nk, kv * dim, dtype, gap)
        self.lse = Mat(nq, heads, "f32")
        dev = lambda a: torch.as_tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        self.a = iso.Attn(q=self.q.view, k=self.k.view, v=self.v.view, ld_q=self.q.ld, ld_k=self.k.ld, ld_v=self.v.ld,
                          start_q=dev(self.at_q), start_k=dev(self.at_k), sequences=len(lens_q), tokens_q=nq, tokens_k=nk,
                          heads=heads, heads_kv=kv, dim=dim, scale=self.scale, out=self.out.view, ld_out=self.out.ld,
                          lse=self.lse.view, causal=causal, window=window, dout=self.dout.view, ld_dout=self.dout.ld,
                          dq=self.dq.view, dk=self.dk.view, dv=self.dv.view, ld_dq=self.dq.ld, ld_dk=self.dk.ld, ld_dv=self.dv.ld)

    def forward(self, ws=None, stream=None):
        ws = iso.attend_workspace(self.a, code(self.dtype)) if ws is None else ws
        iso.iso_attend(self.a, code(self.dtype), ws=ws, stream=stream)
        return ws

    def backward(self, ws=None, stream=None):
        ws = iso.attend_workspace(self.a, code(self.dtype), grad=True) if ws is None else ws
        iso.iso_attend_grad(self.a, code(self.dtype), ws=ws, stream=stream)
        return ws

    def parts(self):
        """(rows, keys, columns of the head, its kv columns, head) of every sequence and head."""
        group = self.heads // self.kv
        for s in range(len(self.lens_q)):
            for h in range(self.heads):
                yield (slice(self.at_q[s], self.at_q[s + 1]), slice(self.at_k[s], self.at_k[s + 1]),
                       slice(h * self.dim, (h + 1) * self.dim), slice(h // group * self.dim, (h // group + 1) * self.dim), h)

    def seen(self, n, m):
        see = np.zeros((n, m), dtype=bool)
        for i in range(n):
            lo, hi = gr.keys_seen(i, n, m, self.causal, self.window)
            see[i, lo:hi] = True
        return see

    def _outside(self, x, at, name):
        assert (x[:at[0]] == 7.25).all() and (x[at[-1]:] == 7.25).all(), f"{name}: rows of no sequence were written"

    def check_forward(self):
        u, ur = unit(self.dtype), 2.0 ** -8 if self.dtype == "bf16" else 0.0
        out, lse = self.out.host(), self.lse.host()
        self._outside(out, self.at_q, "out"), self._outside(lse, self.at_q, "lse")
        for rows, keys, c, e, h in self.parts():
            q, k, v = self.host["q"][rows, c], self.host["k"][keys, e], self.host["v"][keys, e]
            want, l = gr.attend(q, k, v, self.scale, self.causal, self.window)
            see = self.seen(len(q), len(k))
            with np.errstate(all="ignore"):
                a = np.where(see, self.scale * np.abs(q) @ np.abs(k).T, 0.0)
                p = np.where(see, np.exp(np.where(see, self.scale * q @ k.T, 0.0) - l[:, None]), 0.0)
                ep = ((self.dim + 8) * E24 * (a + 1)).max(1, initial=0.0) + (self.dim + 8) * E24 * np.where(np.isfinite(l), np.abs(l), 0)
                err = 2 * ep + (len(k) + 8) * E24
                mass = p @ np.where(np.isfinite(v), np.abs(v), 0.0)
                close(out[rows, c], want, SLACK * ((err + ur)[:, None] * mass + u * np.abs(want)))
                close(lse[rows, h], l, SLACK * err)

    def check_backward(self):
        u, ur = unit(self.dtype), 2.0 ** -8 if self.dtype == "bf16" else 0.0
        got = [self.dq.host(), self.dk.host(), self.dv.host()]
        for x, at, name in zip(got, (self.at_q, self.at_k, self.at_k), ("dq", "dk", "dv")):
            self._outside(x, at, name)
        out, lse = self.out.host(), self.lse.host()
        want = [np.zeros(x.shape) for x in got]
        tol = [np.zeros(x.shape) for x in got]
        for rows, keys, c, e, h in self.parts():
            q, k, v = self.host["q"][rows, c], self.host["k"][keys, e], self.host["v"][keys, e]
            o, do, l = out[rows, c], self.host["dout"][rows, c], lse[rows, h]
            n, m = len(q), len(k)
            dq, dk, dv = gr.attend_grad(q, k, v, o, l, do, self.scale, self.causal, self.window)
            want[0][rows, c], want[1][keys, e], want[2][keys, e] = dq, want[1][keys, e] + dk, want[2][keys, e] + dv
            see = self.seen(n, m)
            with np.errstate(all="ignore"):
                z = lambda x: np.where(np.isfinite(x), x, 0.0)  # noqa: E731
                q, k, v, o, do, l0 = z(q), z(k), z(v), z(o), z(do), z(l)
                p = np.where(see, np.exp(self.scale * q @ k.T - l0[:, None]), 0.0)
                ep = (self.dim + 8) * E24 * (self.scale * np.abs(q) @ np.abs(k).T + np.abs(l0)[:, None] + 1)
                delta = (do * o).sum(1, keepdims=True)
                ds = p * (do @ v.T - delta)
                edp = (self.dim + 8) * E24 * (np.abs(do) @ np.abs(v).T + (np.abs(do) * np.abs(o)).sum(1, keepdims=True))
                eds = np.abs(ds) * (ep + ur + (max(n * self.heads // self.kv, m) + 8) * E24) + p * edp
                edv = p * (ep + ur + (n * self.heads // self.kv + 8) * E24)
                tol[0][rows, c] = self.scale * eds @ np.abs(k)
                if ur and m:
                    widest = np.stack([np.abs(k)[see[i]].max(0, initial=0.0) for i in range(n)]) if n else np.zeros((0, self.dim))
                    tol[0][rows, c] += self.scale * ur * np.abs(ds).sum(1, keepdims=True) * widest
                tol[1][keys, e] += self.scale * eds.T @ np.abs(q)
                tol[2][keys, e] += edv.T @ np.abs(do)
        for x, w, t, at in zip(got, want, tol, (self.at_q, self.at_k, self.at_k)):
            s = slice(at[0], at[-1])
            with np.errstate(all="ignore"):
                close(x[s], w[s], SLACK * (t[s] + u * np.abs(w[s])) + 2.0 ** -126)
